// Launches that overlap the end of what precedes them on their stream.
#pragma once
#include <cuda_runtime.h>

namespace cmsd {
namespace {

// Waits for the end of the launch before, then lets the next one of the stream take
// its place on the GPU: the first thing in a kernel of an early launch.  (The other
// way about, whole calls would queue up on the SMs behind one another: a gradient of
// 32768 rows in a graph of such calls took 51 us instead of 32.)  Such a kernel
// has no read-only loads (__ldg): what it reads may be written while its CTAs are
// already there, and the wait orders ordinary loads alone.
__device__ __forceinline__ void wait_for_previous() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
// a launch that may begin before what precedes it on the stream has ended (early)
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
