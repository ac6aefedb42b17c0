// Error words of the operators' kernels.
#pragma once
#include <cuda_runtime.h>

#include <mutex>

namespace cmsd {

// What a kernel finds goes to its workspace's word and to one of the device (for
// each translation unit), which outlives a workspace that nobody kept.
namespace {
__device__ unsigned g_errors, g_taken;
__device__ __forceinline__ void report(unsigned* word, unsigned bits) {
  if (word) atomicOr(word, bits);                    // (null: a call without a workspace)
  atomicOr(&g_errors, bits);
}
__global__ void take_errors_kernel() { g_taken = atomicExch(&g_errors, 0u); }
// the current device's word, which is cleared; s is waited for
cudaError_t take_errors(unsigned* flags, cudaStream_t s) {
  static std::mutex mu;                              // (one reader of g_taken at a time)
  std::lock_guard<std::mutex> lk(mu);
  take_errors_kernel<<<1, 1, 0, s>>>();
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbolAsync(flags, g_taken, sizeof(unsigned), 0, cudaMemcpyDeviceToHost, s);
  const cudaError_t f = cudaStreamSynchronize(s);    // (whatever e is: flags is the caller's)
  return e != cudaSuccess ? e : f;
}
}  // namespace

}  // namespace cmsd
