// Launches that overlap the end of what precedes them on their stream.
#pragma once
#include <cuda_runtime.h>

namespace cmsd {
namespace {

// a launch that may begin before what precedes it on the stream has ended (early:
// the first launch of a call does not)
template <typename... P, typename... A>
cudaError_t launch(bool early, void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t s,
                   A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Dynamic shared memory above 48 KB, once for each kernel (its own `done`) and device.
template <typename K>
cudaError_t allow_smem(K kernel, size_t smem, unsigned long long* done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = 1ull << (dev & 63);
  if (__atomic_load_n(done, __ATOMIC_ACQUIRE) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) __atomic_fetch_or(done, bit, __ATOMIC_ACQ_REL);
  return e;
}

}  // namespace
}  // namespace cmsd
