// Scaled rows of the token table (include/cmsd.h, cmsd_embedding) and the
// table's gradient (cmsd_embedding_backward).
#include <cuda_bf16.h>

#include <mutex>

#include "cmsd_device.cuh"
#include "cmsd_errors.cuh"
#include "cmsd_rows.cuh"
#include "cmsd_train.h"

namespace cmsd {
namespace {

constexpr int kThreads = 128;

// a CTA a row
template <typename T>
__global__ void __launch_bounds__(kThreads) embed_kernel(const EmbedArgs a) {
  for (int r = blockIdx.x; r < a.R; r += gridDim.x) {
    const int token = a.tokens[r];
    const bool in = token >= 0 && token < a.V;
    const bool keep = in && token != a.ignore;
    if (!in && token != a.ignore && threadIdx.x == 0) report(nullptr, 1u);
    T* x = static_cast<T*>(a.x) + (size_t)r * a.d;
    const T* row = static_cast<const T*>(a.table) + (size_t)(keep ? token : 0) * a.d;
    for (int j = threadIdx.x; j < a.d; j += kThreads) x[j] = from_float<T>(keep ? to_float(row[j]) * a.scale : 0.f);
  }
}

// a CTA an entry of the vocabulary: looks its rows up in all tokens, in order
template <typename T>
__global__ void __launch_bounds__(kThreads) embed_backward_kernel(const EmbedArgs a) {
  __shared__ int s_hit[kThreads / 32];
  if (blockIdx.x == 0)
    for (int r = threadIdx.x; r < a.R; r += kThreads) {
      const int token = a.tokens[r];
      if (token != a.ignore && (token < 0 || token >= a.V)) report(a.err, 1u);
    }
  for (int v = blockIdx.x; v < a.V; v += gridDim.x) {
    T* out = static_cast<T*>(a.d_table) + (size_t)v * a.d;
    for (int j0 = 0; j0 < a.d; j0 += kThreads) {
      const int j = j0 + threadIdx.x;
      float sum = 0.f;
      bool any = false;
      for (int r0 = 0; r0 < a.R && v != a.ignore; r0 += kThreads) {
        const int r = r0 + threadIdx.x;
        const unsigned hit = __ballot_sync(kFull, r < a.R && a.tokens[r] == v);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) s_hit[threadIdx.x >> 5] = (int)hit;
        __syncthreads();
        for (int w = 0; w < kThreads / 32; ++w)
          for (unsigned m = (unsigned)s_hit[w]; m; m &= m - 1) {
            any = true;
            if (j < a.d) sum += to_float(static_cast<const T*>(a.d_x)[(size_t)(r0 + 32 * w + __ffs((int)m) - 1) * a.d + j]);
          }
      }
      if (j < a.d && (any || !a.add)) out[j] = from_float<T>(sum * a.scale + (a.add ? to_float(out[j]) : 0.f));
    }
  }
}

}  // namespace

size_t embed_layout(EmbedArgs& a, char* w) {
  a.err = (unsigned*)w;
  return 256;
}
cudaError_t take_embed_errors(unsigned* flags, cudaStream_t s) { return take_errors(flags, s); }

cudaError_t launch_embed(const EmbedArgs& a, cudaStream_t s) {
  const unsigned grid = a.R < (1 << 20) ? a.R : 1 << 20;
  if (a.dtype == 0) embed_kernel<float><<<grid, kThreads, 0, s>>>(a);
  else embed_kernel<__nv_bfloat16><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}
cudaError_t launch_embed_backward(const EmbedArgs& a, cudaStream_t s) {
  const unsigned grid = a.V < (1 << 20) ? a.V : 1 << 20;
  if (a.dtype == 0) embed_backward_kernel<float><<<grid, kThreads, 0, s>>>(a);
  else embed_backward_kernel<__nv_bfloat16><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace cmsd
