// Rows as symmetric 8-bit integers (include/cmsd.h, cmsd_quantize_rows) and
// the product of the LM head in 8-bit integers (cmsd_lmhead_i8).
#include <cuda_bf16.h>

#include "cmsd_device.cuh"
#include "cmsd_head.h"

namespace cmsd {
namespace {

// ---- rows as 8-bit integers ---------------------------------------------------
constexpr int kQuantThreads = 256;

// 127 x / a rounded to the nearest whole number, ties to the even one, exactly:
// the quotient by r ~ 1 / a decides unless it lies within 2^-12 of a tie (it is
// off by less than 127 * 2^-21); there the sign of 127 x - c a, c the tie, does,
// from the two products' roundings (each product's error is one fma, and the
// difference of the rounded products is exact, as they are within a factor of
// two of each other).  0 <= x <= a, both scaled so that nothing overflows.
__device__ __forceinline__ float quantize_abs(float x, float a, float r) {
  const float hi = __fmul_rn(127.f, x);
  const float t = hi * r;
  float q = rintf(t);
  const float f = fabsf(t - q);
  if (f > 0.5f - 0x1p-12f) {
    const float k = floorf(t), c = k + 0.5f;
    const float lo = __fmaf_rn(127.f, x, -hi);
    const float ph = __fmul_rn(c, a), pl = __fmaf_rn(c, a, -ph);
    const float past = (hi - ph) + (lo - pl);
    const bool odd = ((int)k & 1) != 0;
    q = past > 0.f || (past == 0.f && odd) ? k + 1.f : k;
  }
  return q;
}

__device__ __forceinline__ float load_f(const float* p, size_t i) { return p[i]; }
__device__ __forceinline__ float load_f(const __nv_bfloat16* p, size_t i) { return __bfloat162float(p[i]); }

template <typename T>
__global__ void __launch_bounds__(kQuantThreads) quantize_kernel(const T* __restrict__ x, int R, int d,
                                                                 int8_t* __restrict__ q, float* __restrict__ scale) {
  __shared__ uint32_t s_max[kQuantThreads / 32];
  const int tid = threadIdx.x;
  for (int r = blockIdx.x; r < R; r += gridDim.x) {
    const T* row = x + (size_t)r * d;
    // the bits of |x| order like its value, an infinity and then NaNs on top
    uint32_t m = 0;
    for (int j = tid; j < d; j += kQuantThreads) m = max(m, __float_as_uint(load_f(row, j)) & 0x7FFFFFFFu);
    m = __reduce_max_sync(kFull, m);
    if ((tid & 31) == 0) s_max[tid >> 5] = m;
    __syncthreads();
    for (int w = 0; w < kQuantThreads / 32; ++w) m = max(m, s_max[w]);
    __syncthreads();
    const float a0 = __uint_as_float(m);
    const bool fine = m != 0 && m < 0x7F800000u;
    const float f = a0 < 0x1p-60f ? 0x1p100f : (a0 > 0x1p60f ? 0x1p-100f : 1.f);
    const float a = fine ? a0 * f : 1.f, inv = 1.f / a;
    for (int j = tid; j < d; j += kQuantThreads) {
      const float v = load_f(row, j);
      const float u = fine ? quantize_abs(fabsf(v) * f, a, inv) : 0.f;
      q[(size_t)r * d + j] = (int8_t)(int)copysignf(u, v);
    }
    if (tid == 0) scale[r] = __fdiv_rn(a0, 127.f);
  }
}

// ---- the product: one thread per four logits of a row ---------------------------
constexpr int kSimpleT = 64;
template <bool kBf16>
__global__ void __launch_bounds__(256) head_i8_kernel(const HeadI8Args a) {
  __shared__ int8_t sh[kSimpleT][20], sw[kSimpleT][20];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int v0 = blockIdx.x * kSimpleT;
  for (int r0 = blockIdx.y * kSimpleT; r0 < a.R; r0 += gridDim.y * kSimpleT) {
    int acc[4][4] = {};
    for (int k = 0; k < a.d; k += 16) {
      const int i = tid >> 2, c = (tid & 3) * 4;
      int h = 0, w = 0;
      if (r0 + i < a.R) h = *reinterpret_cast<const int*>(a.hidden + (size_t)(r0 + i) * a.d + k + c);
      if (v0 + i < a.V) w = *reinterpret_cast<const int*>(a.weight + (size_t)(v0 + i) * a.d + k + c);
      __syncthreads();
      *reinterpret_cast<int*>(&sh[i][c]) = h;
      *reinterpret_cast<int*>(&sw[i][c]) = w;
      __syncthreads();
#pragma unroll
      for (int c4 = 0; c4 < 16; c4 += 4)
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int t = 0; t < 4; ++t)
            acc[u][t] = __dp4a(*reinterpret_cast<const int*>(&sh[ty * 4 + u][c4]),
                               *reinterpret_cast<const int*>(&sw[tx + 16 * t][c4]), acc[u][t]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int r = r0 + ty * 4 + u, v = v0 + tx + 16 * t;
        if (r < a.R && v < a.V) {
          const float z = (float)acc[u][t] * a.hidden_scale[r] * a.weight_scale[v];
          if (kBf16)
            reinterpret_cast<__nv_bfloat16*>(a.logits)[(size_t)r * a.V + v] = __float2bfloat16_rn(z);
          else
            reinterpret_cast<float*>(a.logits)[(size_t)r * a.V + v] = z;
        }
      }
  }
}
}  // namespace

cudaError_t launch_quantize_rows(const void* x, int dtype, int R, int d, int8_t* q, float* scale, cudaStream_t s) {
  const int grid = R < (1 << 20) ? R : 1 << 20;
  if (dtype == 0)
    quantize_kernel<float><<<grid, kQuantThreads, 0, s>>>((const float*)x, R, d, q, scale);
  else
    quantize_kernel<__nv_bfloat16><<<grid, kQuantThreads, 0, s>>>((const __nv_bfloat16*)x, R, d, q, scale);
  return cudaGetLastError();
}

cudaError_t launch_head_i8(const HeadI8Args& a, cudaStream_t s) {
  const int ry = (a.R + kSimpleT - 1) / kSimpleT;
  const dim3 grid((unsigned)((a.V + kSimpleT - 1) / kSimpleT), (unsigned)(ry < 65535 ? ry : 65535));
  if (a.dtype == 0)
    head_i8_kernel<false><<<grid, 256, 0, s>>>(a);
  else
    head_i8_kernel<true><<<grid, 256, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace cmsd
