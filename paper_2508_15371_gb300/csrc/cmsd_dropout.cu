// Dropout from the counter-based generator (include/cmsd.h, cmsd_dropout and
// cmsd_dropout_backward).
//
// A counter's four words are eight entries' bits: one generator call for 16 bytes
// of bf16.  Sixteen bits an entry, not 32, because the generator would bound the
// call otherwise (2^27 bf16 entries without a residual: 78.0 us, 6.9 TB/s; with a
// word an entry 110.7 us, 4.9 TB/s), at rates that are multiples of 2^-16; the kept
// entries' scale is that of the rounded rate.  Bound by memory: R = 16384 d = 2048 bf16
// with a residual 30.4 us, 6.6 TB/s; without 22.1, 6.1.
#include <cuda_bf16.h>

#include "cmsd_device.cuh"
#include "cmsd_launch.cuh"
#include "cmsd_philox.cuh"
#include "cmsd_rows.cuh"
#include "cmsd_train.h"

namespace cmsd {
namespace {

constexpr int kThreads = 256;
constexpr int kEach = 2;                             // counters of a thread, requested together

// whether entry j of a counter's eight is kept
__device__ __forceinline__ bool kept(const U4& p, int j, uint32_t drop) {
  const uint32_t w = j < 2 ? p.x : (j < 4 ? p.y : (j < 6 ? p.z : p.w));
  return (j & 1 ? w >> 16 : w & 0xFFFFu) >= drop;
}

template <typename T, bool RESIDUAL>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropArgs a) {
  constexpr int kVecs = sizeof(T) / 2, kIn = 8 / kVecs;        // 16-byte vectors of eight entries, entries of one
  using V = RowVec<T, kIn>;
  wait_for_previous();
  const int64_t whole = a.n >> 3;                    // counters with all of their entries
  const int64_t g0 = (int64_t)blockIdx.x * (kThreads * kEach) + threadIdx.x;
  const uint4* x = static_cast<const uint4*>(a.x);
  const uint4* r = static_cast<const uint4*>(a.residual);
  uint4 xv[kEach][kVecs], rv[kEach][kVecs];
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int64_t g = g0 + u * kThreads;
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      if (g < whole) {
        xv[u][k] = __ldcs(x + g * kVecs + k);
        if (RESIDUAL) rv[u][k] = __ldcs(r + g * kVecs + k);
      }
  }
  const uint32_t it = iter_word(a.iteration + (a.step ? *a.step : 0u), kPurposeDropout);
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int64_t g = g0 + u * kThreads;
    if (g * 8 >= a.n) break;
    const U4 p = philox4x32_10({(uint32_t)g, (uint32_t)(g >> 32), a.site, it}, seed_lo(a.seed), seed_hi(a.seed));
    if (g < whole) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        float f[kIn], h[kIn];
        V::get(xv[u][k], f);
        if (RESIDUAL) V::get(rv[u][k], h);
#pragma unroll
        for (int j = 0; j < kIn; ++j) {
          const float y = RESIDUAL ? __fmaf_rn(f[j], a.scale, h[j]) : f[j] * a.scale;
          f[j] = kept(p, k * kIn + j, a.drop) ? y : (RESIDUAL ? h[j] : 0.f);
        }
        static_cast<uint4*>(a.y)[g * kVecs + k] = V::put(f);
      }
    } else {                                         // the last entries
      for (int j = 0; j < (int)(a.n & 7); ++j) {
        const int64_t e = g * 8 + j;
        const float h = RESIDUAL ? to_float(static_cast<const T*>(a.residual)[e]) : 0.f;
        const float f = to_float(static_cast<const T*>(a.x)[e]);
        const float y = RESIDUAL ? __fmaf_rn(f, a.scale, h) : f * a.scale;
        static_cast<T*>(a.y)[e] = from_float<T>(kept(p, j, a.drop) ? y : h);
      }
    }
  }
}

template <typename T>
cudaError_t launch_typed(const DropArgs& a, cudaStream_t s) {
  const int64_t ctas = ((a.n + 7) / 8 + kThreads * kEach - 1) / (kThreads * kEach);   // (n < 2^42: below 2^31 of them)
  return launch(true, a.residual ? dropout_kernel<T, true> : dropout_kernel<T, false>, (unsigned)ctas, kThreads, 0, s, a);
}

}  // namespace

cudaError_t launch_dropout(const DropArgs& a, cudaStream_t s) {
  return a.dtype == 0 ? launch_typed<float>(a, s) : launch_typed<__nv_bfloat16>(a, s);
}

}  // namespace cmsd
