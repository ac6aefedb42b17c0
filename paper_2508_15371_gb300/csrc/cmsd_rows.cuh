// Rows of fp32 or bf16 numbers: reading and writing single entries.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

namespace cmsd {

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// entry j of a vector of parameters, float or bf16 (one branch for the whole grid)
__device__ __forceinline__ float param(const void* p, int dtype, int j) {
  return dtype == 0 ? static_cast<const float*>(p)[j] : to_float(static_cast<const __nv_bfloat16*>(p)[j]);
}

}  // namespace cmsd
