// Layer norm (include/cmsd.h, cmsd_layernorm) and its gradients
// (cmsd_layernorm_backward).
//
// Both read each row once: it stays in the registers of its threads between the
// row's sums and what they give.  Bound by memory.
#include <cuda_bf16.h>

#include "cmsd_device.cuh"
#include "cmsd_launch.cuh"
#include "cmsd_rows.cuh"
#include "cmsd_train.h"

namespace cmsd {
namespace {

// VE entries of a vector of parameters, float or bf16 (one branch for the whole grid)
template <int VE>
__device__ __forceinline__ void params(const void* p, int dtype, int j, float (&f)[VE]) {
  if (dtype == 0) {
    const float* q = static_cast<const float*>(p) + j;
    if constexpr (VE % 4 == 0) {
#pragma unroll
      for (int k = 0; k < VE; k += 4) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(q + k));
        f[k] = v.x; f[k + 1] = v.y; f[k + 2] = v.z; f[k + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < VE; ++k) f[k] = __ldg(q + k);
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + j;
    if constexpr (VE % 4 == 0) {
#pragma unroll
      for (int k = 0; k < VE; k += 4) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(q + k));
        f[k] = bf_lo(v.x); f[k + 1] = bf_hi(v.x); f[k + 2] = bf_lo(v.y); f[k + 3] = bf_hi(v.y);
      }
    } else {
#pragma unroll
      for (int k = 0; k < VE; ++k) f[k] = __uint_as_float((uint32_t)__ldg(q + k) << 16);
    }
  }
}

// the sums of N numbers over W warps (those of one row), in every thread; buf: [W][N] for each use, so that no
// two uses without a barrier between them share one
template <int N, int W>
__device__ __forceinline__ void row_sums(float (&v)[N], float* buf) {
#pragma unroll
  for (int o = 16; o; o >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(kFull, v[k], o);
  if (W == 1) return;
  const int w = (threadIdx.x >> 5) % W;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) buf[w * N + k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = 0.f;
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += buf[j * N + k];
}

// ---- forward ---------------------------------------------------------------------------
// W warps a row, NV vectors of VE entries a thread.  Sums are of differences from
// the row's first entry, so that a mean far from zero cancels before anything is
// rounded, and a row of one number gives exactly bias.
template <typename T, int VE, int NV, int W>
__global__ void __launch_bounds__(W > 8 ? 32 * W : 256) norm_kernel(const NormArgs a) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
  __shared__ float s_sum[W > 1 ? 2 * W : 1];
  const int nvec = a.d / VE, lane = threadIdx.x & 31, t = W == 1 ? lane : threadIdx.x;
  const int64_t row = W == 1 ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  if (row >= a.R) return;                            // (whole warps, and none that a barrier waits for)
  const Raw* x = static_cast<const Raw*>(a.x) + (size_t)row * nvec;
  Raw* y = static_cast<Raw*>(a.y) + (size_t)row * nvec;
  Raw raw[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    raw[k] = V::zero();
    if (t + 32 * W * k < nvec) raw[k] = __ldcs(x + t + 32 * W * k);
  }
  const float pilot = to_float(static_cast<const T*>(a.x)[(size_t)row * a.d]);
  float s[1] = {0.f};
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float f[VE];
    V::get(raw[k], f);
    if (t + 32 * W * k < nvec)
#pragma unroll
      for (int j = 0; j < VE; ++j) s[0] += f[j] - pilot;
  }
  row_sums<1, W>(s, s_sum);
  const float c = s[0] / a.d;
  s[0] = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float f[VE];
    V::get(raw[k], f);
    if (t + 32 * W * k < nvec)
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const float h = (f[j] - pilot) - c;
        s[0] = __fmaf_rn(h, h, s[0]);
      }
  }
  row_sums<1, W>(s, s_sum + W);
  const float rstd = 1.f / sqrtf(s[0] / a.d + a.eps);
  if (t == 0) {
    if (a.mean) a.mean[row] = pilot + c;
    if (a.rstd) a.rstd[row] = rstd;
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = t + 32 * W * k;
    if (v >= nvec) continue;
    float f[VE], w[VE], b[VE];
    V::get(raw[k], f);
    if (a.weight) params<VE>(a.weight, a.wdtype, v * VE, w);
    if (a.bias) params<VE>(a.bias, a.wdtype, v * VE, b);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      f[j] = ((f[j] - pilot) - c) * rstd;
      if (a.weight) f[j] *= w[j];
      if (a.bias) f[j] += b[j];
    }
    y[v] = V::put(f);
  }
}

// rows that do not fit: a CTA a row, read three times (from L2)
constexpr int kWide = 1024;
template <typename T>
__global__ void __launch_bounds__(kWide) norm_wide_kernel(const NormArgs a) {
  __shared__ float s_sum[2 * kWide / 32];
  const T* x = static_cast<const T*>(a.x) + (size_t)blockIdx.x * a.d;
  T* y = static_cast<T*>(a.y) + (size_t)blockIdx.x * a.d;
  const float pilot = to_float(x[0]);
  float s[1] = {0.f};
  for (int j = threadIdx.x; j < a.d; j += kWide) s[0] += to_float(x[j]) - pilot;
  row_sums<1, kWide / 32>(s, s_sum);
  const float c = s[0] / a.d;
  s[0] = 0.f;
  for (int j = threadIdx.x; j < a.d; j += kWide) {
    const float h = (to_float(x[j]) - pilot) - c;
    s[0] = __fmaf_rn(h, h, s[0]);
  }
  row_sums<1, kWide / 32>(s, s_sum + kWide / 32);
  const float rstd = 1.f / sqrtf(s[0] / a.d + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[blockIdx.x] = pilot + c;
    if (a.rstd) a.rstd[blockIdx.x] = rstd;
  }
  for (int j = threadIdx.x; j < a.d; j += kWide) {
    float h = ((to_float(x[j]) - pilot) - c) * rstd;
    if (a.weight) h *= param(a.weight, a.wdtype, j);
    if (a.bias) h += param(a.bias, a.wdtype, j);
    y[j] = from_float<T>(h);
  }
}

// ---- gradients ---------------------------------------------------------------------------
// A thread has the same eight columns in all of its rows and keeps their two sums
// over rows in registers; W warps a row, kGroups rows at a time in a CTA, rows_at_once
// of them requested together.  The CTAs' sums (kParts of them at most) are joined by
// norm_join_kernel, in the order of the CTAs.
constexpr int kCols = 8;                             // columns of a thread
__host__ __device__ constexpr int rows_at_once(int w) { return w > 16 ? 1 : 2; }
constexpr int kParts = 456;
template <typename T, int VE, int W>
__global__ void __launch_bounds__(W > 8 ? 32 * W : 256, W > 8 ? 1 : 3) norm_backward_kernel(const NormArgs a) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
  constexpr int NV = kCols / VE, kGroups = W > 8 ? 1 : 8 / W, kRows = rows_at_once(W);
  __shared__ float s_sum[W > 1 ? 2 * kGroups * W * 2 * kRows : 1];
  const int nvec = a.d / VE, t = threadIdx.x % (32 * W), group = threadIdx.x / (32 * W);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  float w[NV][VE], dw[NV][VE], db[NV][VE];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      w[k][j] = 1.f;
      dw[k][j] = db[k][j] = 0.f;
    }
    if (a.weight && t + 32 * W * k < nvec) params<VE>(a.weight, a.wdtype, (t + 32 * W * k) * VE, w[k]);
  }
  const float over_d = 1.f / a.d;
  int turn = 0;
  const int64_t step = (int64_t)gridDim.x * kGroups * kRows;
  for (int64_t r0 = ((int64_t)blockIdx.x * kGroups) * kRows; r0 < a.R; r0 += step, turn ^= 1) {
    Raw xr[kRows][NV], gr[kRows][NV];
    float mean[kRows], rstd[kRows], s[2 * kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t row = r0 + u * kGroups + group;
      const bool in = row < a.R;
      mean[u] = in ? __ldg(a.mean_in + row) : 0.f;
      rstd[u] = in ? __ldg(a.rstd_in + row) : 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int v = t + 32 * W * k;
        xr[u][k] = gr[u][k] = V::zero();
        if (in && v < nvec) {
          xr[u][k] = __ldcs(static_cast<const Raw*>(a.x) + (size_t)row * nvec + v);
          gr[u][k] = __ldcs(static_cast<const Raw*>(a.d_y) + (size_t)row * nvec + v);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      s[2 * u] = s[2 * u + 1] = 0.f;
      const bool in = r0 + u * kGroups + group < a.R;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float x[VE], g[VE];
        V::get(xr[u][k], x);
        V::get(gr[u][k], g);
        if (in && t + 32 * W * k < nvec)
#pragma unroll
          for (int j = 0; j < VE; ++j) {
            const float h = (x[j] - mean[u]) * rstd[u], gw = g[j] * w[k][j];
            dw[k][j] = __fmaf_rn(g[j], h, dw[k][j]);
            db[k][j] += g[j];
            s[2 * u] += gw;
            s[2 * u + 1] = __fmaf_rn(gw, h, s[2 * u + 1]);
          }
      }
    }
    if (a.d_x) {                                      // (the same in the whole grid)
      row_sums<2 * kRows, W>(s, s_sum + (W > 1 ? (turn * kGroups + group) * W * 2 * kRows : 0));
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int64_t row = r0 + u * kGroups + group;
        const float m1 = s[2 * u] * over_d, m2 = s[2 * u + 1] * over_d;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int v = t + 32 * W * k;
          if (row >= a.R || v >= nvec) continue;
          float x[VE], g[VE];
          V::get(xr[u][k], x);
          V::get(gr[u][k], g);
#pragma unroll
          for (int j = 0; j < VE; ++j) {
            const float h = (x[j] - mean[u]) * rstd[u];
            g[j] = rstd[u] * ((g[j] * w[k][j] - m1) - h * m2);
          }
          static_cast<Raw*>(a.d_x)[(size_t)row * nvec + v] = V::put(g);
        }
      }
    }
  }
  if (!a.d_weight && !a.d_bias) return;
  // the groups' sums, in their order
  __shared__ float s_col[kGroups > 1 ? 256 * kCols : 1];
  float* part = a.part + (size_t)blockIdx.x * 2 * a.d;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (kGroups > 1) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < VE; ++j)
          s_col[(group * kCols + k * VE + j) * 32 * W + t] = which ? db[k][j] : dw[k][j];
      __syncthreads();
    }
    if (group == 0)
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (t + 32 * W * k < nvec)
#pragma unroll
          for (int j = 0; j < VE; ++j) {
            float v = which ? db[k][j] : dw[k][j];
            if (kGroups > 1)
              for (int q = 1; q < kGroups; ++q) v += s_col[(q * kCols + k * VE + j) * 32 * W + t];
            part[which * a.d + (t + 32 * W * k) * VE + j] = v;
          }
  }
}

// a CTA 32 columns of one of the two, a warp every eighth of the parts
__global__ void __launch_bounds__(256) norm_join_kernel(const NormArgs a, int parts) {
  __shared__ float s_part[8][32];
  const int j = blockIdx.x * 32 + (threadIdx.x & 31), which = blockIdx.y, warp = threadIdx.x >> 5;
  void* out = which ? a.d_bias : a.d_weight;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (!out) return;
  float v = 0.f;
  if (j < a.d)
#pragma unroll 8
    for (int p = warp; p < parts; p += 8) v += __ldcg(a.part + ((size_t)p * 2 + which) * a.d + j);
  s_part[warp][threadIdx.x & 31] = v;
  __syncthreads();
  if (warp || j >= a.d) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) v += s_part[k][threadIdx.x];
  if (a.wdtype == 0) static_cast<float*>(out)[j] = v;
  else static_cast<__nv_bfloat16*>(out)[j] = __float2bfloat16_rn(v);
}

// rows of over kWideCols columns: d_x by a CTA a row, the sums over rows by a CTA 32 columns
constexpr int kWideCols = 8192;
template <typename T>
__global__ void __launch_bounds__(kWide) norm_wide_dx_kernel(const NormArgs a) {
  __shared__ float s_sum[2 * kWide / 32];
  const size_t at = (size_t)blockIdx.x * a.d;
  const T* x = static_cast<const T*>(a.x) + at;
  const T* dy = static_cast<const T*>(a.d_y) + at;
  const float mean = a.mean_in[blockIdx.x], rstd = a.rstd_in[blockIdx.x], over_d = 1.f / a.d;
  float s[2] = {0.f, 0.f};
  for (int j = threadIdx.x; j < a.d; j += kWide) {
    const float g = to_float(dy[j]) * (a.weight ? param(a.weight, a.wdtype, j) : 1.f);
    s[0] += g;
    s[1] = __fmaf_rn(g, (to_float(x[j]) - mean) * rstd, s[1]);
  }
  row_sums<2, kWide / 32>(s, s_sum);
  const float m1 = s[0] * over_d, m2 = s[1] * over_d;
  for (int j = threadIdx.x; j < a.d; j += kWide) {
    const float g = to_float(dy[j]) * (a.weight ? param(a.weight, a.wdtype, j) : 1.f);
    const float h = (to_float(x[j]) - mean) * rstd;
    static_cast<T*>(a.d_x)[at + j] = from_float<T>(rstd * ((g - m1) - h * m2));
  }
}
template <typename T>
__global__ void __launch_bounds__(256) norm_wide_sums_kernel(const NormArgs a) {
  __shared__ float s_w[8][32], s_b[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = blockIdx.x * 32 + lane;
  float w = 0.f, b = 0.f;
  if (j < a.d)
#pragma unroll 8
    for (int64_t r = (int64_t)blockIdx.y * 8 + warp; r < a.R; r += (int64_t)gridDim.y * 8) {
      const float g = to_float(static_cast<const T*>(a.d_y)[(size_t)r * a.d + j]);
      w = __fmaf_rn(g, (to_float(static_cast<const T*>(a.x)[(size_t)r * a.d + j]) - a.mean_in[r]) * a.rstd_in[r], w);
      b += g;
    }
  s_w[warp][lane] = w;
  s_b[warp][lane] = b;
  __syncthreads();
  if (warp || j >= a.d) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) {
    w += s_w[k][lane];
    b += s_b[k][lane];
  }
  float* part = a.part + (size_t)blockIdx.y * 2 * a.d;
  part[j] = w;
  part[a.d + j] = b;
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
// warps of a row in norm_backward_kernel: kCols columns a thread
int row_warps(int d) {
  int w = 1;
  while (w * 32 * kCols < d) w *= 2;
  return w;
}
// CTAs whose sums over rows are joined, by R and d alone
int part_count(int R, int d) {
  if (d > kWideCols) return R < 64 * 8 ? ceil_div(R, 8) : 64;
  const int w = row_warps(d), at_once = (w > 8 ? 1 : 8 / w) * rows_at_once(w), most = w > 16 ? kParts / 3 : (w > 8 ? kParts / 3 * 2 : kParts);
  const int n = ceil_div(R, at_once);
  return n < most ? n : most;
}

template <typename T, int VE>
cudaError_t launch_rows(const NormArgs& a, cudaStream_t s) {
  const auto one = [&](auto kernel) {
    // a warp a CTA until every SM has two, then four
    const int warps = a.R <= 304 ? 1 : 4;
    kernel<<<ceil_div(a.R, warps), 32 * warps, 0, s>>>(a);
    return cudaGetLastError();
  };
  const auto many = [&](auto kernel, int threads) {
    kernel<<<a.R, threads, 0, s>>>(a);
    return cudaGetLastError();
  };
  if (a.d <= 256) return one(norm_kernel<T, VE, 8 / VE, 1>);
  if (a.d <= 512) return one(norm_kernel<T, VE, 16 / VE, 1>);
  if (a.d <= 1024) return one(norm_kernel<T, VE, 32 / VE, 1>);
  if (a.d <= 2048) return one(norm_kernel<T, VE, 64 / VE, 1>);
  if (a.d <= 4096) return many(norm_kernel<T, VE, 16 / VE, 8>, 256);
  if (a.d <= 8192) return many(norm_kernel<T, VE, 32 / VE, 8>, 256);
  if (a.d <= 32768) return many(norm_kernel<T, VE, 32 / VE, 32>, 1024);
  return many(norm_wide_kernel<T>, kWide);
}

template <typename T, int VE>
cudaError_t launch_gradients(const NormArgs& a, int parts, cudaStream_t s) {
  const auto go = [&](auto kernel, int threads) {
    kernel<<<parts, threads, 0, s>>>(a);
    return cudaGetLastError();
  };
  switch (row_warps(a.d)) {
    case 1: return go(norm_backward_kernel<T, VE, 1>, 256);
    case 2: return go(norm_backward_kernel<T, VE, 2>, 256);
    case 4: return go(norm_backward_kernel<T, VE, 4>, 256);
    case 8: return go(norm_backward_kernel<T, VE, 8>, 256);
    case 16: return go(norm_backward_kernel<T, VE, 16>, 512);
    default: return go(norm_backward_kernel<T, VE, 32>, 1024);
  }
}
template <typename T>
cudaError_t launch_wide_gradients(const NormArgs& a, int parts, cudaStream_t s) {
  if (a.d_x) norm_wide_dx_kernel<T><<<a.R, kWide, 0, s>>>(a);
  if (a.d_weight || a.d_bias) norm_wide_sums_kernel<T><<<dim3(ceil_div(a.d, 32), parts), 256, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace

size_t norm_layout(NormArgs& a, char* w) {
  a.part = (float*)w;
  const size_t n = (size_t)part_count(a.R > 0 ? a.R : 1, a.d) * 2 * a.d * 4;
  return (n + 255) / 256 * 256;
}

cudaError_t launch_norm(const NormArgs& a, cudaStream_t s) {
  return by_row_type(a.dtype, a.d, [&](auto t) { return launch_rows<typename decltype(t)::T, decltype(t)::VE>(a, s); });
}

cudaError_t launch_norm_backward(const NormArgs& a, cudaStream_t s) {
  const int parts = part_count(a.R, a.d);
  cudaError_t e;
  if (a.d > kWideCols)
    e = a.dtype == 0 ? launch_wide_gradients<float>(a, parts, s) : launch_wide_gradients<__nv_bfloat16>(a, parts, s);
  else
    e = by_row_type(a.dtype, a.d, [&](auto t) {
      return launch_gradients<typename decltype(t)::T, decltype(t)::VE>(a, parts, s);
    });
  if (e != cudaSuccess || (!a.d_weight && !a.d_bias)) return e;
  return launch(true, norm_join_kernel, dim3(ceil_div(a.d, 32), 2), 256, 0, s, a, parts);
}

}  // namespace cmsd
