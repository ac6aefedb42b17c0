// Rows of fp32 or bf16 numbers: entries, and vectors of VE entries as the rows'
// alignment allows (16 bytes; 4 bytes of bf16; one entry).
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "cmsd_device.cuh"

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

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}

// VE entries of type T: the words that one load or store moves, and their values
template <typename T, int VE>
struct RowVec;
template <>
struct RowVec<float, 4> {
  using Raw = uint4;
  static __device__ __forceinline__ Raw zero() { return make_uint4(0, 0, 0, 0); }
  static __device__ __forceinline__ void get(const Raw& r, float (&f)[4]) {
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ Raw put(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <>
struct RowVec<float, 1> {
  using Raw = float;
  static __device__ __forceinline__ Raw zero() { return 0.f; }
  static __device__ __forceinline__ void get(const Raw& r, float (&f)[1]) { f[0] = r; }
  static __device__ __forceinline__ Raw put(const float (&f)[1]) { return f[0]; }
};
template <>
struct RowVec<__nv_bfloat16, 8> {
  using Raw = uint4;
  static __device__ __forceinline__ Raw zero() { return make_uint4(0, 0, 0, 0); }
  static __device__ __forceinline__ void get(const Raw& r, float (&f)[8]) {
    f[0] = bf_lo(r.x); f[1] = bf_hi(r.x); f[2] = bf_lo(r.y); f[3] = bf_hi(r.y);
    f[4] = bf_lo(r.z); f[5] = bf_hi(r.z); f[6] = bf_lo(r.w); f[7] = bf_hi(r.w);
  }
  static __device__ __forceinline__ Raw put(const float (&f)[8]) {
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  }
};
template <>
struct RowVec<__nv_bfloat16, 2> {
  using Raw = uint32_t;
  static __device__ __forceinline__ Raw zero() { return 0; }
  static __device__ __forceinline__ void get(const Raw& r, float (&f)[2]) { f[0] = bf_lo(r); f[1] = bf_hi(r); }
  static __device__ __forceinline__ Raw put(const float (&f)[2]) { return pack_bf16(f[0], f[1]); }
};
template <>
struct RowVec<__nv_bfloat16, 1> {
  using Raw = uint16_t;
  static __device__ __forceinline__ Raw zero() { return 0; }
  static __device__ __forceinline__ void get(const Raw& r, float (&f)[1]) { f[0] = __uint_as_float((uint32_t)r << 16); }
  static __device__ __forceinline__ Raw put(const float (&f)[1]) { return (uint16_t)pack_bf16(f[0], 0.f); }
};
// VE entries (an even number) as pairs for the packed fp32 instructions
template <typename T, int VE>
__device__ __forceinline__ void get_pairs(const typename RowVec<T, VE>::Raw& r, u64 (&p)[VE / 2]) {
  if constexpr (sizeof(T) == 2 && VE == 8) {
    p[0] = bf2_to_f2(r.x); p[1] = bf2_to_f2(r.y); p[2] = bf2_to_f2(r.z); p[3] = bf2_to_f2(r.w);
  } else {
    float f[VE];
    RowVec<T, VE>::get(r, f);
#pragma unroll
    for (int j = 0; j < VE / 2; ++j) p[j] = pack2(f[2 * j], f[2 * j + 1]);
  }
}
template <typename T, int VE>
__device__ __forceinline__ typename RowVec<T, VE>::Raw put_pairs(const u64 (&p)[VE / 2]) {
  float f[VE];
#pragma unroll
  for (int j = 0; j < VE / 2; ++j) {
    f[2 * j] = lo32f(p[j]);
    f[2 * j + 1] = hi32f(p[j]);
  }
  return RowVec<T, VE>::put(f);
}

// f(RowType<T, VE>) with the widest vectors that every row of d entries begins on
template <typename T_, int VE_>
struct RowType {
  using T = T_;
  static constexpr int VE = VE_;
};
template <typename F>
cudaError_t by_row_type(int dtype, int d, F&& f) {
  if (dtype == 0) return d % 4 == 0 ? f(RowType<float, 4>()) : f(RowType<float, 1>());
  if (d % 8 == 0) return f(RowType<__nv_bfloat16, 8>());
  return d % 2 == 0 ? f(RowType<__nv_bfloat16, 2>()) : f(RowType<__nv_bfloat16, 1>());
}

}  // namespace cmsd
