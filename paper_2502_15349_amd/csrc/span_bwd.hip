// Backward pass of span attention: the launch in front of its main kernels, the dispatch to these, and the spans of packed documents.
#include "span_bwd.hpp"

#include "launch.hpp"
#include "span_documents.hpp"

namespace ae {
namespace {

// In what order the tiles of 128 rows of batch entry b are walked: those with the longest walk first, on either side, equal ones as they would come
// otherwise.  Their lengths are taken from the first and the last row of every 32 (whatever they are, the order holds every tile once).  A workgroup beside those
// that form delta.  Documents leave walks of very different lengths, and the last ones decide:
// 1 x 32/8 x 8192 in four documents 761 us as they come, 630 in this order (192/128 869, 763; 64/64 406, 398), 1 x 16 x 4000 166, 153 (152, 151; 80, 76); among
// many workgroups 1 % longer (4 x 32/8 x 4096 712, 719).
__device__ void order_tiles(const BwdSpanParams& p, const SpanPrepare& w, int b) {
  typedef __attribute__((ext_vector_type(4))) int i32x4;
  __shared__ __attribute__((aligned(16))) int32_t first[4 * kMostOrdered], behind[4 * kMostOrdered], cost[2 * kMostOrdered];
  constexpr int kNone = 0x7fffffff;
  const int nk = (p.L_k + 127) / 128, nq = (p.L_q + 127) / 128, off = p.L_k - p.L_q;
#pragma unroll
  for (int n = 0; n < 4 * kMostOrdered / 256; ++n) {  // (four for each tile: those of rows that there are not see nothing)
    const int k = 256 * n + (int)threadIdx.x;
    int lo0, hi0, lo1, hi1;
    span_of(w.span, b, min(32 * k, p.L_q - 1), off, p.L_k, lo0, hi0);
    span_of(w.span, b, min(32 * k + 31, p.L_q - 1), off, p.L_k, lo1, hi1);
    first[k] = 32 * k < p.L_q ? min(lo0 < hi0 ? lo0 : kNone, lo1 < hi1 ? lo1 : kNone) : kNone;
    behind[k] = 32 * k < p.L_q ? max(hi0, hi1) : 0;
  }
  __syncthreads();
  const int t = (int)threadIdx.x < nk ? (int)threadIdx.x : (int)threadIdx.x - kMostOrdered;  // threads [0, nk): key tiles, from kMostOrdered on: query tiles
  const bool key = (int)threadIdx.x < nk, query = t >= 0 && !key && t < nq;
  if (key) {
    int f = 4 * nq, e = 0;
#pragma unroll 4
    for (int k = 0; k < nq; ++k) {
      const i32x4 lo = *reinterpret_cast<const i32x4*>(first + 4 * k), hi = *reinterpret_cast<const i32x4*>(behind + 4 * k);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const bool meets = lo[x] < 128 * t + 128 && hi[x] > 128 * t;
        f = min(f, meets ? 4 * k + x : 4 * nq);
        e = meets ? 4 * k + x + 1 : e;
      }
    }
    cost[t] = max(e - f, 0);
  } else if (query) {
    int f = kNone, e = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) f = min(f, first[4 * t + x]), e = max(e, behind[4 * t + x]);
    cost[kMostOrdered + t] = e > 0 ? e - f : 0;
  } else if (t < 0) {
    cost[threadIdx.x] = -1;
  } else {
    cost[kMostOrdered + t] = -1;
  }
  __syncthreads();
  if (!key && !query) return;
  const int32_t* of = cost + (key ? 0 : kMostOrdered);
  const int mine = of[t], n = key ? nk : nq;
  int place = 0;
#pragma unroll 4
  for (int k = 0; k < (n + 3) / 4; ++k) {
    const i32x4 c = *reinterpret_cast<const i32x4*>(of + 4 * k);
#pragma unroll
    for (int x = 0; x < 4; ++x) place += c[x] > mine || (c[x] == mine && (key ? 4 * k + x < t : 4 * k + x > t));
  }
  w.order[(int64_t)b * (nk + nq) + (key ? 0 : nk) + place] = t;
}

// Workgroups [0, span_blocks): 256 rows of the spans each; then, where wanted, the order of a batch entry's tiles each; the others: delta, as attn_bwd_delta_kernel forms it (a group of D_v / 8
// lanes owns a row, four passes in flight).  Both only stream.
constexpr int kPasses = 4;
template <int DV>
__global__ __launch_bounds__(256) void span_prepare_kernel(const BwdSpanParams p, const SpanPrepare w, int span_blocks, int order_blocks) {
  const int lane = threadIdx.x & 63;
  if ((int)blockIdx.x >= span_blocks && (int)blockIdx.x < span_blocks + order_blocks) return order_tiles(p, w, (int)blockIdx.x - span_blocks);
  if ((int)blockIdx.x < span_blocks) {
    const int per = (p.L_q + 255) / 256, b = (int)blockIdx.x / per, i = (int)blockIdx.x % per * 256 + (int)threadIdx.x;
    constexpr int kNone = 0x7fffffff;
    int lo = 0, hi = 0;
    if (i < p.L_q) {
      span_of(w.span, b, i, p.L_k - p.L_q, p.L_k, lo, hi);
      w.begin[(int64_t)b * p.L_q + i] = lo;
      w.end[(int64_t)b * p.L_q + i] = hi;
    }
    const bool there = i < p.L_q;
    SpanBlock s{lo < hi ? lo : kNone, hi, lo, there ? hi : kNone};
#pragma unroll
    for (int k = 1; k < 32; k *= 2) {
      s.first = min(s.first, __shfl_xor(s.first, k));
      s.behind = max(s.behind, __shfl_xor(s.behind, k));
      s.last_lo = max(s.last_lo, __shfl_xor(s.last_lo, k));
      s.least_hi = min(s.least_hi, __shfl_xor(s.least_hi, k));
    }
    if (there && (lane & 31) == 0) w.blocks[(int64_t)b * ((p.L_q + 31) / 32) + i / 32] = s;
    return;
  }
  constexpr int LPR = DV / 8, RPP = 64 / LPR, RPW = RPP * kPasses;  // lanes per row, rows per pass, rows per wavefront
  const int64_t rows = (int64_t)p.B * p.H_q * p.L_q;
  const int sub = lane % LPR;
  const int64_t r0 = ((int64_t)(blockIdx.x - span_blocks - order_blocks) * 4 + (threadIdx.x >> 6)) * RPW + lane / LPR;
  bf16x8 g[kPasses];
  f32x4 o[kPasses][2];
#pragma unroll
  for (int k = 0; k < kPasses; ++k) {
    const int64_t r = r0 + k * RPP < rows ? r0 + k * RPP : rows - 1;
    const int i = (int)(r % p.L_q), hq = (int)((r / p.L_q) % p.H_q), b = (int)(r / ((int64_t)p.L_q * p.H_q));
    const int64_t ob = b * p.os[0] + hq * p.os[1] + (int64_t)i * p.os[2] + 8 * sub;
    g[k] = *reinterpret_cast<const bf16x8*>(p.dO + b * p.dos[0] + hq * p.dos[1] + (int64_t)i * p.dos[2] + 8 * sub);
    if (p.o_bf16) {
      const bf16x4 lo = *reinterpret_cast<const bf16x4*>(static_cast<const __bf16*>(p.O) + ob);  // (strides of O are multiples of 4)
      const bf16x4 hi = *reinterpret_cast<const bf16x4*>(static_cast<const __bf16*>(p.O) + ob + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[k][0][e] = (float)lo[e];
        o[k][1][e] = (float)hi[e];
      }
    } else {
      o[k][0] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.O) + ob);
      o[k][1] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.O) + ob + 4);
    }
  }
#pragma unroll
  for (int k = 0; k < kPasses; ++k) {
    float acc = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc += o[k][e / 4][e % 4] * (float)g[k][e];
#pragma unroll
    for (int s = LPR / 2; s >= 1; s >>= 1) acc += __shfl_xor(acc, s);
    const int64_t r = r0 + k * RPP;
    if (r < rows && sub == 0) p.delta[r] = acc;
  }
}

template <int DV>
hipError_t launch_prepare(const BwdSpanParams& p, const SpanPrepare& w, hipStream_t s) {
  constexpr int RPW = 64 / (DV / 8) * kPasses;
  const int64_t rows = (int64_t)p.B * p.H_q * p.L_q, delta = (rows + 4 * RPW - 1) / (4 * RPW), spans = (int64_t)p.B * ((p.L_q + 255) / 256);
  const int64_t orders = w.order != nullptr ? p.B : 0;
  if (!launch_fits(delta + spans + orders, 256) || spans > 0x7fffffff) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(span_prepare_kernel<DV>, dim3((unsigned)(delta + spans + orders)), dim3(256), 0, s, p, w, (int)spans, (int)orders);
  return hipGetLastError();
}

// One thread a token: its document by bisection of the offsets.
__global__ __launch_bounds__(256) void span_documents_kernel(const SpanDocuments p) {
  const int per = (p.L + 255) / 256, b = (int)blockIdx.x / per, i = (int)blockIdx.x % per * 256 + (int)threadIdx.x;
  if (i >= p.L) return;
  const int32_t* at = p.offsets + b * p.offset_stride;
  int lo = 0, hi = 0;
  if (i >= at[0] && i < at[p.n_docs]) {
    int d = 0, behind = p.n_docs;  // at[d] <= i < at[behind]
    while (behind - d > 1) {
      const int mid = (d + behind) / 2;
      if (at[mid] <= i) d = mid;
      else behind = mid;
    }
    const int first = max(at[d], 0), last = min(at[d + 1], p.L);
    const int prefix = p.prefix != nullptr ? max(0, min(p.prefix[b * p.prefix_stride + d], last - first)) : 0;
    lo = first;
    hi = p.kind == SPAN_ALL ? last : max(i + 1, first + prefix);
    if (p.kind == SPAN_WINDOW) lo = max(first, i - p.window + 1);
  }
  p.begin[b * (int64_t)p.L + i] = lo;
  p.end[b * (int64_t)p.L + i] = hi;
}

}  // namespace

hipError_t launch_span_documents(const SpanDocuments& p, hipStream_t s) {
  const int64_t grid = (int64_t)p.B * ((p.L + 255) / 256);
  if (!launch_fits(grid, 256) || grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(span_documents_kernel, dim3((unsigned)grid), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_span_bwd_64_64(const BwdSpanParams&, const DecayTable&, int, hipStream_t);
hipError_t launch_span_bwd_128_128(const BwdSpanParams&, const DecayTable&, int, hipStream_t);
hipError_t launch_span_bwd_192_128(const BwdSpanParams&, const DecayTable&, int, hipStream_t);

hipError_t launch_span_backward(const BwdSpanParams& p, const SpanPrepare& w, const DecayTable& dt, int dqk, int dv, int var, hipStream_t s) {
  const hipError_t e = dv == 64 ? launch_prepare<64>(p, w, s) : launch_prepare<128>(p, w, s);
  if (e != hipSuccess) return e;
  if (dqk == 64) return launch_span_bwd_64_64(p, dt, var, s);
  if (dqk == 128) return launch_span_bwd_128_128(p, dt, var, s);
  return launch_span_bwd_192_128(p, dt, var, s);
}

}  // namespace ae
