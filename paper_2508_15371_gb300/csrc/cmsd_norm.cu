// Layer norm (include/cmsd.h, cmsd_layernorm) and its gradients
// (cmsd_layernorm_backward).
#include <cuda_bf16.h>

#include "cmsd_device.cuh"
#include "cmsd_rows.cuh"
#include "cmsd_train.h"

namespace cmsd {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float cta_sum(float v) {
  __shared__ float s_part[kThreads / 32];
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) v += s_part[w];
  return v;
}

// a CTA a row
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_kernel(const NormArgs a) {
  for (int r = blockIdx.x; r < a.R; r += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + (size_t)r * a.d;
    T* y = static_cast<T*>(a.y) + (size_t)r * a.d;
    // about the row's first entry: exact for a row of one number, and what is far from zero cancels first
    const float pilot = to_float(x[0]);
    float s = 0.f;
    for (int j = threadIdx.x; j < a.d; j += kThreads) s += to_float(x[j]) - pilot;
    const float c = cta_sum(s) / a.d;
    s = 0.f;
    for (int j = threadIdx.x; j < a.d; j += kThreads) {
      const float t = to_float(x[j]) - pilot - c;
      s += t * t;
    }
    const float rstd = 1.f / sqrtf(cta_sum(s) / a.d + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = pilot + c;
      if (a.rstd) a.rstd[r] = rstd;
    }
    for (int j = threadIdx.x; j < a.d; j += kThreads) {
      const float h = (to_float(x[j]) - pilot - c) * rstd;
      y[j] = from_float<T>(h * (a.weight ? param(a.weight, a.wdtype, j) : 1.f) + (a.bias ? param(a.bias, a.wdtype, j) : 0.f));
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) norm_dx_kernel(const NormArgs a) {
  for (int r = blockIdx.x; r < a.R; r += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + (size_t)r * a.d;
    const T* dy = static_cast<const T*>(a.d_y) + (size_t)r * a.d;
    T* dx = static_cast<T*>(a.d_x) + (size_t)r * a.d;
    const float mean = a.mean_in[r], rstd = a.rstd_in[r];
    float s1 = 0.f, s2 = 0.f;
    for (int j = threadIdx.x; j < a.d; j += kThreads) {
      const float g = to_float(dy[j]) * (a.weight ? param(a.weight, a.wdtype, j) : 1.f);
      s1 += g;
      s2 += g * ((to_float(x[j]) - mean) * rstd);
    }
    const float m1 = cta_sum(s1) / a.d, m2 = cta_sum(s2) / a.d;
    for (int j = threadIdx.x; j < a.d; j += kThreads) {
      const float g = to_float(dy[j]) * (a.weight ? param(a.weight, a.wdtype, j) : 1.f);
      dx[j] = from_float<T>(rstd * (g - m1 - (to_float(x[j]) - mean) * rstd * m2));
    }
  }
}

// a CTA 32 columns, eight warps a row each
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_dw_kernel(const NormArgs a) {
  __shared__ float s_w[kThreads], s_b[kThreads];
  const int j = blockIdx.x * 32 + (threadIdx.x & 31);
  float w = 0.f, b = 0.f;
  if (j < a.d)
    for (int r = threadIdx.x >> 5; r < a.R; r += kThreads / 32) {
      const float g = to_float(static_cast<const T*>(a.d_y)[(size_t)r * a.d + j]);
      w += g * ((to_float(static_cast<const T*>(a.x)[(size_t)r * a.d + j]) - a.mean_in[r]) * a.rstd_in[r]);
      b += g;
    }
  s_w[threadIdx.x] = w;
  s_b[threadIdx.x] = b;
  __syncthreads();
  if (threadIdx.x >= 32 || j >= a.d) return;
  w = b = 0.f;
  for (int k = 0; k < kThreads; k += 32) {
    w += s_w[k + threadIdx.x];
    b += s_b[k + threadIdx.x];
  }
  if (a.wdtype == 0) {
    if (a.d_weight) static_cast<float*>(a.d_weight)[j] = w;
    if (a.d_bias) static_cast<float*>(a.d_bias)[j] = b;
  } else {
    if (a.d_weight) static_cast<__nv_bfloat16*>(a.d_weight)[j] = __float2bfloat16_rn(w);
    if (a.d_bias) static_cast<__nv_bfloat16*>(a.d_bias)[j] = __float2bfloat16_rn(b);
  }
}

}  // namespace

size_t norm_layout(NormArgs& a, char* w) {
  a.part = (float*)w;
  return 256;
}

cudaError_t launch_norm(const NormArgs& a, cudaStream_t s) {
  const unsigned grid = a.R < (1 << 20) ? a.R : 1 << 20;
  if (a.dtype == 0) norm_kernel<float><<<grid, kThreads, 0, s>>>(a);
  else norm_kernel<__nv_bfloat16><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_norm_backward(const NormArgs& a, cudaStream_t s) {
  const unsigned grid = a.R < (1 << 20) ? a.R : 1 << 20, cols = (a.d + 31) / 32;
  if (a.d_x && a.R > 0) {
    if (a.dtype == 0) norm_dx_kernel<float><<<grid, kThreads, 0, s>>>(a);
    else norm_dx_kernel<__nv_bfloat16><<<grid, kThreads, 0, s>>>(a);
  }
  if (a.d_weight || a.d_bias) {
    if (a.dtype == 0) norm_dw_kernel<float><<<cols, kThreads, 0, s>>>(a);
    else norm_dw_kernel<__nv_bfloat16><<<cols, kThreads, 0, s>>>(a);
  }
  return cudaGetLastError();
}

}  // namespace cmsd
