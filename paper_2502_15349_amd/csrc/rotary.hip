// Rotary positions, forward and backward.
//
//   y1 = a (x1 cos t - x2 sin t),  y2 = a (x2 cos t + x1 sin t),  t = position * f_i   (backward: t -> -t)
//
// Bound by memory: every element is read and written once, with three operations on it.  What else there is to do is the
// sine and cosine of one angle per (row, pair), the same for every head: a thread owns one piece of a row (a vector of
// pairs) and walks the heads with the sines and cosines in registers, the rows of four heads in flight at a time.
// 4 x 2048 rows of 32 + 8 heads of 128, bf16, heads side by side: 33.8 us, 5.0 TB/s of reads and writes.
//
// The angle: f_i / 2 pi modulo 1 is kept as a 64-bit fraction of a turn, so that position times it, in integers, wraps as
// turns do and nothing is lost at far positions (in 32-bit floats position 10^6 would leave an error of 0.06 radians).  The
// top 32 bits are split into a quadrant and a rest of at most 1/8 turn, for which the Taylor series up to the tenth power
// are exact to 2^-25.
#include "rotary.hpp"

#include <algorithm>

#include "launch.hpp"

namespace ae {
namespace {

// sin and cos of hi / 2^32 turns
__device__ __forceinline__ void turn_sincos(uint32_t hi, float& s, float& c) {
  const uint32_t quad = (hi + 0x20000000u) >> 30;
  const float a = (float)(int32_t)(hi - (quad << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32; |a| <= pi / 4
  const float z = a * a;
  const float sp = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(__builtin_fmaf(z, 2.7557319e-6f, -1.9841270e-4f), z, 8.3333333e-3f), z, -1.6666667e-1f), z * a, a);
  const float cp = __builtin_fmaf(
      __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(__builtin_fmaf(z, -2.7557319e-7f, 2.4801587e-5f), z, -1.3888889e-3f), z, 4.1666667e-2f), z, -0.5f), z, 1.f);
  const float u = quad & 1 ? cp : sp, v = quad & 1 ? sp : cp;
  s = quad & 2 ? -u : u;
  c = (quad + 1) & 2 ? -v : v;
}

template <typename T, int N>
struct Piece {
  T v[N];
} ;

template <typename T, int N>
__device__ __forceinline__ Piece<T, N> load_piece(const T* p) {
  Piece<T, N> r;
  __builtin_memcpy(&r, __builtin_assume_aligned(p, N * sizeof(T)), sizeof(r));
  return r;
}
template <typename T, int N>
__device__ __forceinline__ void store_piece(T* p, const Piece<T, N>& r) {
  __builtin_memcpy(__builtin_assume_aligned(p, N * sizeof(T)), &r, sizeof(r));
}

constexpr int kHeads = 4;  // heads in flight

// VEC: elements of a piece (16 bytes, or one element where rows are not made of whole 16-byte pieces).  A thread has either the
// two pieces of VEC pairs, or one piece of the elements behind rot_dim.
// SIDE: heads of a row that neighbouring threads take.
template <typename T, int VEC, bool INTER, int SIDE>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryParams p, const RotaryTable t) {
  typedef Piece<T, VEC> P;
  const int n_rot = p.half / VEC, pieces = n_rot + (p.D - 2 * p.half) / VEC;
  // pieces of a row fastest, then SIDE heads next to each other, then rows
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row_side = id / pieces, row = row_side / SIDE;
  const int piece = (int)(id - row_side * pieces);
  if (row >= (int64_t)p.B * p.L) return;
  const int b = (int)(row / p.L), l = (int)(row - (int64_t)b * p.L);
  // the thread's heads: h, h + SIDE, ... below h_end
  const int h0 = blockIdx.y * p.heads_per_thread * SIDE, h_end = min(p.H[0] + p.H[1], h0 + p.heads_per_thread * SIDE);
  int h = h0 + (int)(row_side - row * SIDE);

  auto at = [&](int hh, bool out) {  // first element of the row of head hh (Q's heads, then K's)
    const int w = hh >= p.H[0] ? 1 : 0;
    const int64_t(&s)[3] = out ? p.ys[w] : p.xs[w];
    const int64_t o = b * s[0] + (hh - (w ? p.H[0] : 0)) * s[1] + l * s[2];
    return out ? static_cast<T*>(p.y[w]) + o : const_cast<T*>(static_cast<const T*>(p.x[w])) + o;
  };
  if (piece >= n_rot) {  // behind the rotated part
    const int e = 2 * p.half + (piece - n_rot) * VEC;
    for (; h < h_end; h += kHeads * SIDE) {
      P x[kHeads];
#pragma unroll
      for (int u = 0; u < kHeads; ++u) x[u] = load_piece<T, VEC>(at(h + u * SIDE < h_end ? h + u * SIDE : h, false) + e);
#pragma unroll
      for (int u = 0; u < kHeads; ++u)
        if (h + u * SIDE < h_end) store_piece<T, VEC>(at(h + u * SIDE, true) + e, x[u]);
    }
    return;
  }
  const int e1 = INTER ? 2 * VEC * piece : VEC * piece, e2 = INTER ? e1 + VEC : e1 + p.half;
  const int32_t pos = p.positions[b * p.position_stride + l];
  float sn[VEC], cs[VEC];
  bool first = true;
  for (; h < h_end; h += kHeads * SIDE) {
    P x1[kHeads], x2[kHeads];
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {  // (heads past the last repeat the first; all reads before the first write: y may be x)
      const T* x = at(h + u * SIDE < h_end ? h + u * SIDE : h, false);
      x1[u] = load_piece<T, VEC>(x + e1);
      x2[u] = load_piece<T, VEC>(x + e2);
    }
    if (first) {  // behind the first loads: a call of few rows is a chain of latencies
      first = false;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        // the top half of pos * turn (64 bits, modulo 1): pos as an unsigned number, minus 2^32 turns' worth where it is negative
        const uint64_t f = t.turn[VEC * piece + i];
        const uint32_t lo = (uint32_t)f;
        const uint32_t hi = __umulhi((uint32_t)pos, lo) + (uint32_t)pos * (uint32_t)(f >> 32) - (pos < 0 ? lo : 0u);
        turn_sincos(hi, sn[i], cs[i]);
        sn[i] *= p.backward ? -p.amp : p.amp;
        cs[i] *= p.amp;
      }
    }
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      P y1, y2;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        // neighbouring pairs: pair i is elements 2 i, 2 i + 1 of the 2 VEC that the two pieces hold together
        const float a = (float)(INTER ? (2 * i < VEC ? x1[u].v[(2 * i) % VEC] : x2[u].v[(2 * i) % VEC]) : x1[u].v[i]);
        const float c = (float)(INTER ? (2 * i + 1 < VEC ? x1[u].v[(2 * i + 1) % VEC] : x2[u].v[(2 * i + 1) % VEC]) : x2[u].v[i]);
        const T o1 = (T)__builtin_fmaf(a, cs[i], -c * sn[i]), o2 = (T)__builtin_fmaf(c, cs[i], a * sn[i]);
        if constexpr (INTER) {
          (2 * i < VEC ? y1 : y2).v[(2 * i) % VEC] = o1;
          (2 * i + 1 < VEC ? y1 : y2).v[(2 * i + 1) % VEC] = o2;
        } else {
          y1.v[i] = o1;
          y2.v[i] = o2;
        }
      }
      if (h + u * SIDE < h_end) {
        T* y = at(h + u * SIDE, true);
        store_piece<T, VEC>(y + e1, y1);
        store_piece<T, VEC>(y + e2, y2);
      }
    }
  }
}

template <typename T, int VEC, int SIDE>
hipError_t launch_side(RotaryParams p, const RotaryTable& t, hipStream_t s) {
  const int heads = p.H[0] + p.H[1];
  const int64_t items = (int64_t)p.B * p.L * SIDE * (p.half / VEC + (p.D - 2 * p.half) / VEC);
  const int64_t bx = (items + 255) / 256;
  // Heads per thread: as many as leave 2048 workgroups (eight for each compute unit), a multiple of those in flight.
  int hpt = kHeads;
  while (hpt < 16 && hpt * SIDE < heads && bx * ((heads + 2 * hpt * SIDE - 1) / (2 * hpt * SIDE)) >= 2048) hpt *= 2;
  p.heads_per_thread = hpt;
  const int by = (heads + hpt * SIDE - 1) / (hpt * SIDE);
  if (by > 65535 || !launch_fits(bx * by, 256)) return hipErrorInvalidConfiguration;
  if (p.interleaved) hipLaunchKernelGGL((rotary_kernel<T, VEC, true, SIDE>), dim3((unsigned)bx, by), dim3(256), 0, s, p, t);
  else hipLaunchKernelGGL((rotary_kernel<T, VEC, false, SIDE>), dim3((unsigned)bx, by), dim3(256), 0, s, p, t);
  return hipGetLastError();
}

// Neighbouring lanes take neighbouring memory: some heads of a row where heads are the closer ones (rows of all heads side by
// side, as a fused projection leaves them), else rows of a head.  4 x 2048 rows of 32 + 8 heads of 128, side by side, bf16: 42.7 us with 1
// head, 34.0 with 4, 35.9 with 8; 16 x 1500 rows of 64 + 8 heads, fp32: 368, 338, 316.
template <typename T, int VEC>
hipError_t launch(const RotaryParams& p, const RotaryTable& t, hipStream_t s) {
  constexpr int kSide = sizeof(T) == 4 ? 8 : 4;
  if (p.xs[0][1] < p.xs[0][2] && p.H[0] + p.H[1] >= kSide) return launch_side<T, VEC, kSide>(p, t, s);
  return launch_side<T, VEC, 1>(p, t, s);
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& p, const RotaryTable& t, bool wide, hipStream_t s) {
  if (p.f32) return wide ? launch<float, 4>(p, t, s) : launch<float, 1>(p, t, s);
  return wide ? launch<__bf16, 8>(p, t, s) : launch<__bf16, 1>(p, t, s);
}

}  // namespace ae
