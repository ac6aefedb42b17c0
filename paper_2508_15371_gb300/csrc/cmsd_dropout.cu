// Dropout from the counter-based generator (include/cmsd.h, cmsd_dropout and
// cmsd_dropout_backward).
#include <cuda_bf16.h>

#include "cmsd_device.cuh"
#include "cmsd_philox.cuh"
#include "cmsd_rows.cuh"
#include "cmsd_train.h"

namespace cmsd {
namespace {

constexpr int kThreads = 256;

// a thread the eight entries of one counter
template <typename T>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropArgs a) {
  const uint32_t it = iter_word(a.iteration + (a.step ? *a.step : 0u), kPurposeDropout);
  const int64_t groups = (a.n + 7) / 8;
  for (int64_t g = blockIdx.x * (int64_t)kThreads + threadIdx.x; g < groups; g += (int64_t)gridDim.x * kThreads) {
    const U4 p = philox4x32_10({(uint32_t)g, (uint32_t)(g >> 32), a.site, it}, seed_lo(a.seed), seed_hi(a.seed));
    for (int j = 0; j < 8; ++j) {
      const int64_t e = 8 * g + j;
      if (e >= a.n) break;
      const uint32_t w = j < 2 ? p.x : (j < 4 ? p.y : (j < 6 ? p.z : p.w));
      const bool keep = (j & 1 ? w >> 16 : w & 0xFFFFu) >= a.drop;
      const float x = keep ? to_float(static_cast<const T*>(a.x)[e]) : 0.f;
      const float r = a.residual ? to_float(static_cast<const T*>(a.residual)[e]) : 0.f;
      static_cast<T*>(a.y)[e] = from_float<T>(keep ? (a.residual ? __fmaf_rn(x, a.scale, r) : x * a.scale) : r);
    }
  }
}

}  // namespace

cudaError_t launch_dropout(const DropArgs& a, cudaStream_t s) {
  const int64_t ctas = ((a.n + 7) / 8 + kThreads - 1) / kThreads;
  const unsigned grid = (unsigned)(ctas < (1 << 20) ? ctas : 1 << 20);
  if (a.dtype == 0) dropout_kernel<float><<<grid, kThreads, 0, s>>>(a);
  else dropout_kernel<__nv_bfloat16><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace cmsd
