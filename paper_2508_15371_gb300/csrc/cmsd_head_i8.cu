// Rows as symmetric 8-bit integers (include/cmsd.h, cmsd_quantize_rows) and
// the product of the LM head in 8-bit integers (cmsd_lmhead_i8).
#include <cuda_bf16.h>

#include "cmsd_head.h"
#include "cmsd_tc.cuh"

namespace cmsd {
namespace {

// four 8-bit integers as fp16 (two pairs), exactly
__device__ __forceinline__ void i8_to_half(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const uint32_t u = w ^ 0x80808080u;               // byte + 128
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(__byte_perm(u, 0x64646464u, 0x4140)), "r"(0x64806480u));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(__byte_perm(u, 0x64646464u, 0x4342)), "r"(0x64806480u));
}

// ---- rows as 8-bit integers ---------------------------------------------------
//
// One pass: a row's numbers stay in the registers of its warp (or of the eight
// warps of a CTA for wide rows) between the search for the largest and the
// rounding, so memory, 2 or 4 bytes read and one written per number, bounds it
// (R=128256 d=2048: bf16 117 us, 6.7 TB/s; f32 186 us, 7.1 TB/s).

// 127 x / a rounded to the nearest whole number, ties to the even one, exactly,
// where an approximation t of the quotient is within 2^-12 of a tie: the sign of
// 127 x - c a, c the tie, decides, from the two products' roundings (each
// product's error is one fma, and the difference of the rounded products is
// exact, as they are within a factor of two of each other).  0 <= x <= a, both
// scaled so that nothing overflows.
__device__ __noinline__ float quantize_abs(float x, float a) {
  const float hi = __fmul_rn(127.f, x);
  const float t = __fdividef(hi, a);
  const float q = rintf(t);
  if (fabsf(t - q) <= 0.5f - 0x1p-12f) return q;
  const float k = floorf(t), c = k + 0.5f;
  const float lo = __fmaf_rn(127.f, x, -hi);
  const float ph = __fmul_rn(c, a), pl = __fmaf_rn(c, a, -ph);
  const float past = (hi - ph) + (lo - pl);
  const bool odd = ((int)k & 1) != 0;
  return past > 0.f || (past == 0.f && odd) ? k + 1.f : k;
}

template <typename T>
struct QuantVec;                                    // 16 bytes of a row
template <>
struct QuantVec<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ float get(const uint4& v, int j) {
    return __uint_as_float(j == 0 ? v.x : (j == 1 ? v.y : (j == 2 ? v.z : v.w)));
  }
  static __device__ __forceinline__ uint32_t mag(const uint4& v) {
    return max(max(v.x & 0x7FFFFFFFu, v.y & 0x7FFFFFFFu), max(v.z & 0x7FFFFFFFu, v.w & 0x7FFFFFFFu));
  }
};
template <>
struct QuantVec<__nv_bfloat16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ float get(const uint4& v, int j) {
    const uint32_t w = j < 2 ? v.x : (j < 4 ? v.y : (j < 6 ? v.z : v.w));
    return j & 1 ? bf_hi(w) : bf_lo(w);
  }
  static __device__ __forceinline__ uint32_t mag(const uint4& v) {
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu),
                                __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
    return max(m & 0xFFFF0000u, m << 16);
  }
};

struct QuantRow {
  float a, f, k, kl;     // largest magnitude scaled by f; 127 / a and what rounding it left out
  bool fine, plain;      // finite and not zero; no scaling needed
};
// the bits of |x| order like its value, an infinity and then NaNs on top
__device__ __forceinline__ QuantRow quant_row(uint32_t m) {
  QuantRow r;
  const float a0 = __uint_as_float(m);
  r.fine = m != 0 && m < 0x7F800000u;
  r.plain = a0 >= 0x1p-60f && a0 <= 0x1p60f;
  r.f = r.plain ? 1.f : (a0 < 1.f ? 0x1p100f : 0x1p-100f);
  r.a = r.fine ? a0 * r.f : 1.f;
  r.k = 127.f / r.a;
  r.kl = __fmaf_rn(-r.k, r.a, 127.f) / r.a;
  return r;
}
// One 16-byte vector as kN bytes in words o[0 .. kN / 4).  x k rounded by adding
// 1.5 * 2^23; the distance of x (k + kl) from it, exact to 2^-24, shows a tie.
// Ties of bf16 numbers are common (every x = a / 2 is one) and stand apart:
// with x = X 2^e, a = A 2^f, X and A below 256 and f - e <= 8, 127 x / a is a tie
// or at least 2^-7 / (2 A) > 2^-17 from one.  Ties of fp32 numbers are rare, but
// others lie as near, and an exact comparison decides.
template <typename T>
__device__ __forceinline__ void quant_vec(const uint4& v, const QuantRow& r, uint32_t* o) {
  using Q = QuantVec<T>;
  constexpr float kMagic = 12582912.f;              // 1.5 * 2^23
  constexpr float kTie = Q::kN == 8 ? 0.5f - 0x1p-18f : 0.5f - 0x1p-22f;
  uint32_t y[Q::kN];
  float off = 1.f;
  if (r.plain) {
    off = 0.f;
#pragma unroll
    for (int j = 0; j < Q::kN; ++j) {
      const float x = Q::get(v, j);
      const float s = __fmaf_rn(x, r.k, kMagic);
      off = fmaxf(off, fabsf(__fmaf_rn(x, r.kl, __fmaf_rn(x, r.k, kMagic - s))));
      y[j] = __float_as_uint(s);
    }
  }
  if (off > kTie) {
    if (Q::kN == 8 && r.plain) {
#pragma unroll
      for (int j = 0; j < Q::kN; ++j) {             // k + 1/2: half of it is a quarter from the even one's half
        const float x = Q::get(v, j), q = __uint_as_float(y[j]) - kMagic;
        const float even = 2.f * rintf(0.5f * (x * r.k));
        if (fabsf(__fmaf_rn(x, r.kl, __fmaf_rn(x, r.k, -q))) > kTie) y[j] = __float_as_uint(even + kMagic);
      }
    } else {
#pragma unroll 1
      for (int j = 0; j < Q::kN; ++j) {
        const float x = Q::get(v, j);
        const float q = r.fine ? quantize_abs(fabsf(x) * r.f, r.a) : 0.f;
        const uint32_t b = (uint32_t)(int)copysignf(q, x);
#pragma unroll
        for (int u = 0; u < Q::kN; ++u) y[u] = u == j ? b : y[u];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < Q::kN / 4; ++j)
    o[j] = __byte_perm(__byte_perm(y[4 * j], y[4 * j + 1], 0x0040), __byte_perm(y[4 * j + 2], y[4 * j + 3], 0x0040),
                       0x5410);
}
template <typename T>
__device__ __forceinline__ void quant_store(int8_t* dst, const uint32_t* o) {
  if (QuantVec<T>::kN == 8)
    *reinterpret_cast<uint2*>(dst) = make_uint2(o[0], o[1]);
  else
    *reinterpret_cast<uint32_t*>(dst) = o[0];
}

constexpr int kQuantThreads = 128;                  // four rows of a warp each
constexpr int kQuantWide = 256;                     // one row
// Rows of up to 32 * NV vectors, a warp kRows of them at once: short rows alone
// leave too little in flight (R=128256 d=512 bf16 58 us with one, 39 with four).
template <typename T, int NV, int kRows>
__global__ void __launch_bounds__(kQuantThreads) quantize_warp_kernel(const T* __restrict__ x, int R, int d,
                                                                      int8_t* __restrict__ q, float* __restrict__ scale) {
  constexpr int kN = QuantVec<T>::kN;
  const int lane = threadIdx.x & 31, vecs = d / kN;
  const int64_t r0 = ((int64_t)blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5)) * kRows;
  const int rows = (int)min((int64_t)kRows, R - r0);
  if (rows <= 0) return;
  const uint4* src = reinterpret_cast<const uint4*>(x + (size_t)r0 * d);
  uint4 v[kRows][NV];
#pragma unroll
  for (int k = 0; k < kRows; ++k)
#pragma unroll
    for (int i = 0; i < NV; ++i)
      v[k][i] = k < rows && lane + 32 * i < vecs ? ld_stream(src + k * vecs + lane + 32 * i) : make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    if (k >= rows) return;
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) m = max(m, QuantVec<T>::mag(v[k][i]));
    m = __reduce_max_sync(kFull, m);
    const QuantRow row = quant_row(m);
    int8_t* dst = q + (size_t)(r0 + k) * d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      uint32_t o[kN / 4];
      quant_vec<T>(v[k][i], row, o);
      if (lane + 32 * i < vecs) quant_store<T>(dst + (lane + 32 * i) * kN, o);
    }
    if (lane == 0) scale[r0 + k] = __fdiv_rn(__uint_as_float(m), 127.f);
  }
}
// wider rows, a CTA each: up to kQuantWide * NV vectors in registers, what lies
// beyond is read twice
template <typename T, int NV>
__global__ void __launch_bounds__(kQuantWide) quantize_cta_kernel(const T* __restrict__ x, int R, int d,
                                                                  int8_t* __restrict__ q, float* __restrict__ scale) {
  constexpr int kN = QuantVec<T>::kN;
  __shared__ uint32_t s_max[2][kQuantWide / 32];
  const int tid = threadIdx.x, vecs = d / kN;
  int turn = 0;
  for (int r = blockIdx.x; r < R; r += gridDim.x, turn ^= 1) {
    const uint4* src = reinterpret_cast<const uint4*>(x + (size_t)r * d);
    uint4 v[NV];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      v[i] = tid + kQuantWide * i < vecs ? ld_stream(src + tid + kQuantWide * i) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NV; ++i) m = max(m, QuantVec<T>::mag(v[i]));
    for (int i = tid + kQuantWide * NV; i < vecs; i += kQuantWide) m = max(m, QuantVec<T>::mag(src[i]));
    m = __reduce_max_sync(kFull, m);
    if ((tid & 31) == 0) s_max[turn][tid >> 5] = m;  // (two arrays in turn: one barrier a row)
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kQuantWide / 32; ++w) m = max(m, s_max[turn][w]);
    const QuantRow row = quant_row(m);
    int8_t* dst = q + (size_t)r * d;
    uint32_t o[kN / 4];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      quant_vec<T>(v[i], row, o);
      if (tid + kQuantWide * i < vecs) quant_store<T>(dst + (tid + kQuantWide * i) * kN, o);
    }
    for (int i = tid + kQuantWide * NV; i < vecs; i += kQuantWide) {
      quant_vec<T>(src[i], row, o);
      quant_store<T>(dst + i * kN, o);
    }
    if (tid == 0) scale[r] = __fdiv_rn(__uint_as_float(m), 127.f);
  }
}

template <typename T>
cudaError_t launch_quantize(const T* x, int R, int d, int8_t* q, float* scale, cudaStream_t s) {
  const int vecs = d / QuantVec<T>::kN;
  auto ctas = [&](int per_warp) {
    const int64_t per = kQuantThreads / 32 * per_warp;
    return (unsigned)((R + per - 1) / per);
  };
  // Several rows a warp where enough CTAs are left to fill the SMs (us with and
  // without.  Four rows, bf16 d=512: R=2048 3.3, 2.7; 4096 3.6, 3.5; 8192 4.7, 5.3;
  // 65536 20, 30.  Two rows, bf16 d=1024: R=16384 10.7, 10.5; 32768 17.8, 17.9; 65536
  // 33.2, 35.5; f32 d=512: 8192 4.0, 3.9; 32768 12.0, 12.3; 65536 21.0, 21.8)
  if (vecs <= 32 * 2 && R >= 8192)
    quantize_warp_kernel<T, 2, 4><<<ctas(4), kQuantThreads, 0, s>>>(x, R, d, q, scale);
  else if (vecs <= 32 * 4 && R >= 32768)
    quantize_warp_kernel<T, 4, 2><<<ctas(2), kQuantThreads, 0, s>>>(x, R, d, q, scale);
  else if (vecs <= 32 * 4)
    quantize_warp_kernel<T, 4, 1><<<ctas(1), kQuantThreads, 0, s>>>(x, R, d, q, scale);
  else if (vecs <= 32 * 8)
    quantize_warp_kernel<T, 8, 1><<<ctas(1), kQuantThreads, 0, s>>>(x, R, d, q, scale);
  else if (vecs <= 32 * 16)
    quantize_warp_kernel<T, 16, 1><<<ctas(1), kQuantThreads, 0, s>>>(x, R, d, q, scale);
  else if (vecs <= kQuantWide * 4)
    quantize_cta_kernel<T, 4><<<(unsigned)(R < (1 << 20) ? R : 1 << 20), kQuantWide, 0, s>>>(x, R, d, q, scale);
  else
    quantize_cta_kernel<T, 8><<<(unsigned)(R < (1 << 20) ? R : 1 << 20), kQuantWide, 0, s>>>(x, R, d, q, scale);
  return cudaGetLastError();
}

// ---- the product ----------------------------------------------------------------
//
// A whole number of 8 bits is exact in fp16, its products are exact in the
// tensor cores and their sums exact in fp32 up to 2^24.  So the integers go
// through the fp16 tensor cores (GB300's integer tensor rate is far below).
// Where every token of a tile has magnitudes that add up to at most 2^17, as
// rows scaled by their largest do up to a few thousand entries, no sum with
// 8-bit weights passes 2^24 and all of K is summed by the tensor cores; else the
// sums of each 1024 entries (of products of at most 2^14) are added up as 32-bit
// integers, 64 tokens of the tile at a time (the registers hold no more).  Either
// way the sum is exact.  (R=512 d=2048 V=128256: 166 us with one sum, the tensor pipe
// 76 % busy; R=64 50 us, 5.6 TB/s.)  Only the 8-bit weight is read from memory; its bytes
// become fp16 on their way into tensor memory, where the MMA takes its A from:
// byte + 128 is placed into the low mantissa bits of 1024.0, and 1152 is
// subtracted, both exact.
//
// The MMA's M is the vocabulary: a pair of CTAs (cta_group::2) with up to 128
// entries each, so that a stage of the tokens (N, up to 192 of them, half in each
// CTA) is read from L2 once for both.  Each CTA:
//   warp 0       lane 0 fills a ring with 128 bytes of K of its weight rows;
//   warp 2       lane 0 another with its half of the tokens' (fp16, from the
//                workspace), counted at the first CTA's barriers;
//   warp 1       of the first CTA: one lane issues the MMAs of both;
//   warps 4..11  turn the weight into fp16 in tensor memory: thread = 64 of K of
//                one entry;
//   warps 12..19 add up, scale and write the sums: thread = one entry, every
//                second group of 16 tokens.
// Barriers: wfull / wempty (TMA <-> fp16), hfull / hempty (TMA <-> MMA), afull /
// aempty (fp16 <-> MMA, buffers in tensor memory), dfull / dempty (MMA <-> sums,
// two sets of accumulators).  Every wait is bounded.
constexpr int kI8Rows = 128;                        // vocabulary entries per CTA and tile at most
constexpr int kI8K = 128;                           // K per stage
constexpr int kI8Exact = 1024 / kI8K;               // stages whose sums are exact in fp32 whatever the tokens
constexpr int kI8Threads = 640;
constexpr int kI8WStage = kI8Rows * kI8K;
constexpr int kI8Part = 64;                         // tokens at a time where sums are kept apart
template <int NT>
struct I8Shape {
  static constexpr int kHStage = NT / 2 * kI8K * 2; // this CTA's half of the tokens
  static constexpr int kW = NT == 192 ? 6 : (NT == 128 ? 7 : 8);
  static constexpr int kH = NT == 192 ? 5 : (NT == 128 ? 6 : 8);
  static constexpr int kSum = NT == 192 ? 192 : 128;        // columns of an accumulator
  static constexpr int kA = (512 - 2 * kSum) / 64;  // buffers of the fp16 weight: 64 columns each
  static constexpr int kBars = 2 * kW + 2 * kH + 2 * kA + 4;
  static constexpr size_t kStageBytes = (size_t)kW * kI8WStage + (size_t)kH * kHStage;
  static constexpr size_t kSmem = 1024 + kStageBytes + 8 * kBars + 16;
  static_assert(kSmem <= 227 * 1024, "shared memory");
};
struct I8Plan {
  int height;            // vocabulary entries per CTA and tile
  int cols;              // tokens per tile (a multiple of 32, at most 192)
  int vt, rt;            // tiles (of two CTAs) of the vocabulary and of the tokens
};

// the tokens as fp16, and the sum of each one's magnitudes; a CTA a token
constexpr int kTokenThreads = 128;
__global__ void __launch_bounds__(kTokenThreads) head_i8_tokens_kernel(const HeadI8Args a) {
  __shared__ int s_sum[kTokenThreads / 32];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, vecs = a.d / 16;
  for (int r = blockIdx.x; r < a.R; r += gridDim.x) {
    const uint4* src = reinterpret_cast<const uint4*>(a.hidden + (size_t)r * a.d);
    uint4* dst = reinterpret_cast<uint4*>(a.h16 + (size_t)r * a.d);
    unsigned sum = 0;
    for (int i = tid; i < vecs; i += kTokenThreads) {
      const uint4 x = src[i];
      uint32_t h[8];
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        i8_to_half(w[k], h[2 * k], h[2 * k + 1]);
        sum = __dp4a(__vabsdiffs4(w[k], 0u), 0x01010101u, sum);   // (|-128| is 128)
      }
      dst[2 * i] = make_uint4(h[0], h[1], h[2], h[3]);
      dst[2 * i + 1] = make_uint4(h[4], h[5], h[6], h[7]);
    }
    sum = __reduce_add_sync(kFull, sum);
    if ((tid & 31) == 0) s_sum[tid >> 5] = (int)sum;
    __syncthreads();
    if (tid == 0) {
      int all = 0;
#pragma unroll
      for (int w = 0; w < kTokenThreads / 32; ++w) all += s_sum[w];
      a.mag[r] = all;
    }
    __syncthreads();
  }
}

// Whether a tile of tokens needs the sums of each 1024 entries apart.  Where
// there are several tiles of tokens the next one's magnitudes are requested a tile
// ahead (and not later: the loads are volatile).
struct I8Span {
  int m[6];
  bool is;
  __device__ __forceinline__ void request(const HeadI8Args& a, const I8Plan& p, int t) {
    const int r0 = t % p.rt * p.cols, lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 6; ++i) {
      const int n = lane + 32 * i;
      m[i] = 0;
      if (n < p.cols && r0 + n < a.R)
        asm volatile("ld.global.cg.s32 %0, [%1];" : "=r"(m[i]) : "l"(a.mag + r0 + n) : "memory");
    }
  }
  __device__ __forceinline__ void take() {
    is = __reduce_max_sync(kFull, max(max(max(m[0], m[1]), max(m[2], m[3])), max(m[4], m[5]))) > (1 << 17);
  }
  // the pair's first tile, after the tokens' kernel; each further one
  __device__ __forceinline__ bool first(const HeadI8Args& a, const I8Plan& p, int t, int pairs) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    request(a, p, t);
    take();
    if (p.rt > 1) request(a, p, t + pairs);
    return is;
  }
  __device__ __forceinline__ bool next(const HeadI8Args& a, const I8Plan& p, int t, int pairs) {
    if (p.rt > 1) {
      take();
      request(a, p, t + pairs);
    }
    return is;
  }
};

// map_h, map_p: the tokens in boxes of half a tile, of half a part
template <int NT, bool kBf16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kI8Threads, 1)
    head_i8_kernel(const HeadI8Args a, const I8Plan p, const __grid_constant__ CUtensorMap map_w,
                   const __grid_constant__ CUtensorMap map_h, const __grid_constant__ CUtensorMap map_p) {
  using S = I8Shape<NT>;
  extern __shared__ __align__(1024) unsigned char i8_smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster_rank(), pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  const uint32_t raw = smem_addr(i8_smem);
  const uint32_t base = (raw + 1023u) & ~1023u, hbase = base + S::kW * kI8WStage;
  const uint32_t bars = base + (uint32_t)S::kStageBytes;
  const uint32_t wfull = bars, wempty = wfull + 8 * S::kW;
  const uint32_t hfull = wempty + 8 * S::kW, hempty = hfull + 8 * S::kH;
  const uint32_t afull = hempty + 8 * S::kH, aempty = afull + 8 * S::kA;
  const uint32_t dfull = aempty + 8 * S::kA, dempty = dfull + 16;
  uint32_t* s_taddr = reinterpret_cast<uint32_t*>(i8_smem + (bars - raw) + 8 * S::kBars);
  if (tid == 0) {
    for (int k = 0; k < S::kW; ++k) {
      mbar_init(wfull + 8 * k, 1);
      mbar_init(wempty + 8 * k, 8);
    }
    for (int k = 0; k < S::kH; ++k) {
      mbar_init(hfull + 8 * k, 1);
      mbar_init(hempty + 8 * k, 1);
    }
    for (int b = 0; b < S::kA; ++b) {
      mbar_init(afull + 8 * b, 16);                 // the turning warps of both CTAs
      mbar_init(aempty + 8 * b, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(dfull + 8 * b, 1);
      mbar_init(dempty + 8 * b, 16);                // the summing warps of both CTAs
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(s_taddr)),
                 "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tmem_fence_before();
  cluster_sync_all();
  tmem_fence_after();
  const uint32_t tbase = *s_taddr;                  // two accumulators
  const uint32_t abase = tbase + 2 * S::kSum;       // kA buffers of 64 columns
  const int ks = (a.d + kI8K - 1) / kI8K;           // stages per pass
  const int tiles = p.vt * p.rt;
  const int mine = tiles > pair ? (tiles - pair + pairs - 1) / pairs : 0;
  const int parts = (p.cols + kI8Part - 1) / kI8Part;
  const int part_cols = min(p.cols, kI8Part);
  // A tile takes one pass over K, or one for each part of its tokens.
  I8Span span;
  bool ok = true;

  if (warp == 0) {
    // The weight's first stages do not wait for the tokens' kernel: that one has
    // started, so what precedes it on the stream has ended.
    const uint32_t bytes = (uint32_t)(p.height * kI8K);
    int s = 0, g = 0;
    uint32_t phase = 1;                             // (of the round before: a new barrier's is over)
    for (int i = 0; i < mine; ++i) {
      const int y = ((pair + i * pairs) / p.rt * 2 + rank) * p.height;
      int passes = 1;
      for (int j = 0; j < passes; ++j) {
        if (lane == 0) {
          for (int k = 0; k < ks; ++k, ++g) {
            if (ok) ok = bar_wait<false>(wempty + 8 * s, phase);
            if (!ok) break;
            mbar_arrive_tx(wfull + 8 * s, bytes);
            tma_box(base + s * kI8WStage, &map_w, k * kI8K, y, wfull + 8 * s);
            if (++s == S::kW) {
              s = 0;
              phase ^= 1;
            }
          }
        }
        __syncwarp();
        if (j == 0) {                               // how often the tile's weight is wanted
          const int t = pair + i * pairs;
          passes = (i == 0 ? span.first(a, p, t, pairs) : span.next(a, p, t, pairs)) ? parts : 1;
        }
      }
    }
    g = __shfl_sync(kFull, g, 0);
    // nothing is in flight into this CTA when it ends
    for (int k = (g > S::kW ? g - S::kW : 0); k < g; ++k)
      if (ok) ok = bar_wait<false>(wempty + 8 * (k % S::kW), (uint32_t)((k / S::kW) & 1));
  } else if (warp == 2) {
    const uint32_t hfull0 = map_to(hfull, 0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("fence.proxy.async.global;" ::: "memory");
    int s = 0, g = 0;
    uint32_t phase = 1;
    for (int i = 0; i < mine; ++i) {
      const int t = pair + i * pairs;
      const bool apart = i == 0 ? span.first(a, p, t, pairs) : span.next(a, p, t, pairs);
      const int passes = apart ? parts : 1, cols = apart ? part_cols : p.cols, half = cols / 2;
      const CUtensorMap* map = apart ? &map_p : &map_h;
      for (int j = 0; j < passes; ++j) {
        const int y = t % p.rt * p.cols + j * kI8Part + rank * half;
        if (lane == 0) {
          for (int k = 0; k < ks; ++k, ++g) {
            if (ok) ok = bar_wait<true>(hempty + 8 * s, phase);
            if (!ok) break;
            if (rank == 0) mbar_arrive_tx(hfull + 8 * s, (uint32_t)(cols * kI8K * 2));   // both halves
            const uint32_t dst = hbase + s * S::kHStage;
            tma_box_pair(dst, map, k * kI8K, y, hfull0 + 8 * s);
            tma_box_pair(dst + half * 128, map, k * kI8K + 64, y, hfull0 + 8 * s);
            if (++s == S::kH) {
              s = 0;
              phase ^= 1;
            }
          }
        }
        __syncwarp();
      }
    }
    g = __shfl_sync(kFull, g, 0);
    for (int k = (g > S::kH ? g - S::kH : 0); k < g; ++k)
      if (ok) ok = bar_wait<true>(hempty + 8 * (k % S::kH), (uint32_t)((k / S::kH) & 1));
  } else if (warp == 1) {
    // the whole warp runs through the stages, so that what the MMAs take is
    // formed in uniform registers; one lane issues
    if (rank == 0) {
      const bool leader = elect_lane();
      const uint32_t hempty0 = map_to(hempty, 0), hempty1 = map_to(hempty, 1);
      const uint32_t aempty0 = map_to(aempty, 0), aempty1 = map_to(aempty, 1);
      const uint32_t dfull0 = map_to(dfull, 0), dfull1 = map_to(dfull, 1);
      int c = 0, s = 0, b = 0;                      // sums handed over; ring slot; buffer
      uint32_t phase = 0, aphase = 0;
      for (int i = 0; i < mine; ++i) {
        const int t = pair + i * pairs;
        const bool apart = i == 0 ? span.first(a, p, t, pairs) : span.next(a, p, t, pairs);
        const int len = apart ? min(kI8Exact, ks) : ks, steps = (apart ? parts : 1) * ks;
        const uint32_t cols = (uint32_t)(apart ? part_cols : p.cols);
        const uint32_t idesc = mma_idesc(256, 0, false, false, false) | (cols >> 3) << 17;
        const uint32_t half = cols * 64 >> 4;       // the second 64 of K, in units of 16 bytes
        for (int g = 0, k = 0, part = 0; g < steps; ++g) {
          const int db = c & 1;
          const bool ends = part == len - 1 || k == ks - 1;
          if (part == 0 && c >= 2 && ok) ok = bar_wait<true>(dempty + 8 * db, (uint32_t)((c / 2 - 1) & 1));
          if (ok) ok = bar_wait<true>(hfull + 8 * s, phase);
          if (ok) ok = bar_wait<true>(afull + 8 * b, aphase);
          tmem_fence_after();
          const uint64_t h0 = mma_desc(hbase + s * S::kHStage, 0), h1 = h0 + half;
          const uint32_t d = tbase + db * S::kSum, at = abase + b * 64;
          if (leader && ok) {
#pragma unroll
            for (int j = 0; j < kI8K / 16; ++j)
              mma_pair_tmem_a(d, at + j * 8, (j >> 2 ? h1 : h0) + (uint64_t)(2 * (j & 3)), idesc,
                              j > 0 ? 1u : (uint32_t)(part != 0));
            mma_commit_pair(aempty0 + 8 * b);
            mma_commit_pair(aempty1 + 8 * b);
            mma_commit_pair(hempty0 + 8 * s);
            mma_commit_pair(hempty1 + 8 * s);
            if (ends) {
              mma_commit_pair(dfull0 + 8 * db);
              mma_commit_pair(dfull1 + 8 * db);
            }
          }
          __syncwarp();
          c += ends;
          part = ends ? 0 : part + 1;
          if (++k == ks) k = 0;
          if (++s == S::kH) {
            s = 0;
            phase ^= 1;
          }
          if (++b == S::kA) {
            b = 0;
            aphase ^= 1;
          }
        }
      }
    }
    __syncwarp();
  } else if (warp >= 4 && warp < 12) {
    const int q = warp & 3, half = (warp - 4) >> 2;
    const int row = q * 32 + lane;                  // entry within this CTA's part
    const uint32_t quarter = (uint32_t)(q * 32) << 16;
    const uint32_t wrow = (uint32_t)row * 128, x8 = (uint32_t)(row & 7);
    const uint32_t afull0 = map_to(afull, 0);
    int s = 0, b = 0, g = 0;
    uint32_t phase = 0, aphase = 1;
    // the first pass does not wait for the tokens' kernel
    for (int i = 0, left = mine > 0 ? ks : 0; left > 0;) {
      do {
        if (ok) ok = bar_wait<true>(aempty + 8 * b, aphase);
        if (ok) ok = bar_wait<false>(wfull + 8 * s, phase);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        const uint32_t src = base + s * kI8WStage + wrow;
        uint32_t o[32];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t w0, w1, w2, w3;
          asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                       : "=r"(w0), "=r"(w1), "=r"(w2), "=r"(w3)
                       : "r"(src + (((uint32_t)(4 * half + j) ^ x8) << 4)));
          i8_to_half(w0, o[8 * j], o[8 * j + 1]);
          i8_to_half(w1, o[8 * j + 2], o[8 * j + 3]);
          i8_to_half(w2, o[8 * j + 4], o[8 * j + 5]);
          i8_to_half(w3, o[8 * j + 6], o[8 * j + 7]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive_local(wempty + 8 * s);    // (its bytes are in registers)
        tmem_fence_after();
        tmem_st32(abase + quarter + b * 64 + half * 32, o);
        tmem_st_wait();
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(afull0 + 8 * b);
        if (++s == S::kW) {
          s = 0;
          phase ^= 1;
        }
        if (++b == S::kA) {
          b = 0;
          aphase ^= 1;
        }
        ++g;
      } while (--left > 0);
      if (!ok) break;
      if (g == ks && span.first(a, p, pair, pairs)) left = ks * (parts - 1);
      if (left == 0 && ++i < mine) left = span.next(a, p, pair + i * pairs, pairs) ? ks * parts : ks;
    }
    // the last arrivals at this CTA's barriers are in before it ends
    const int G = g;
    for (g = (G > S::kA ? G - S::kA : 0); g < G; ++g)
      if (ok) ok = bar_wait<true>(aempty + 8 * (g % S::kA), (uint32_t)((g / S::kA) & 1));
  } else if (warp >= 12) {
    const int q = warp & 3, set = (warp - 12) >> 2;
    const int row = q * 32 + lane;
    const uint32_t quarter = (uint32_t)(q * 32) << 16;
    const uint32_t dempty0 = map_to(dempty, 0);
    constexpr int kMine = NT / 32;                  // this set's groups of 16 tokens (every second one)
    const size_t step = (size_t)a.V * (kBf16 ? 2 : 4);
    int c = 0;
    for (int i = 0; i < mine; ++i) {
      const int t = pair + i * pairs;
      const bool apart = i == 0 ? span.first(a, p, t, pairs) : span.next(a, p, t, pairs);
      const int vi = t / p.rt, r0 = (t - vi * p.rt) * p.cols, v = (vi * 2 + rank) * p.height + row;
      const bool in = row < p.height && v < a.V;
      float ws = 0.f, hs[kMine];                    // lane l: the scale of token 32 u + l
#pragma unroll
      for (int u = 0; u < kMine; ++u) hs[u] = __ldg(a.hidden_scale + min(r0 + 32 * u + lane, a.R - 1));
      if (in) ws = __ldg(a.weight_scale + v);
      const int rows = in ? min(a.R - r0, p.cols) : 0;
      // 16 tokens' logits from n on
      auto write = [&](const float (&y)[16], float scales, int n) {
        char* out = reinterpret_cast<char*>(a.logits) + ((size_t)(r0 + n) * a.V + v) * (kBf16 ? 2 : 4);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float h = __shfl_sync(kFull, scales, 16 * set + j);
          if (n + j < rows) {
            const float z = y[j] * h * ws;
            if (kBf16)
              *reinterpret_cast<__nv_bfloat16*>(out) = __float2bfloat16_rn(z);
            else
              *reinterpret_cast<float*>(out) = z;
          }
          out += step;
        }
      };
      auto sum_wait = [&]() {
        if (ok) ok = bar_wait<true>(dfull + 8 * (c & 1), (uint32_t)((c / 2) & 1));
        ok = __all_sync(kFull, ok);
        tmem_fence_after();
      };
      auto sum_done = [&]() {
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(dempty0 + 8 * (c & 1));
        ++c;
      };
      if (!apart) {
        sum_wait();
        if (!ok) break;
        const uint32_t src = tbase + quarter + (c & 1) * S::kSum + 16 * set;
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
          const int n = 16 * (2 * u + set);
          float y[16];
          if (n < p.cols) {
            tmem_ld16_ahead(src + 32 * u, y);
            tmem_ld_wait(y);
          }
          if (n < p.cols && n + 32 >= p.cols) sum_done();     // (this set's last)
          if (n < p.cols) write(y, hs[u], n);
        }
        continue;
      }
      const int len = min(kI8Exact, ks), sums = (ks + len - 1) / len;
#pragma unroll
      for (int j = 0; j < (NT + kI8Part - 1) / kI8Part; ++j) {
        if (j < parts) {
          int acc[2][16];
#pragma unroll
          for (int n = 0; n < 32; ++n) acc[n / 16][n % 16] = 0;
#pragma unroll 1
          for (int k = 0; k < sums; ++k) {
            sum_wait();
            if (!ok) break;
            const uint32_t src = tbase + quarter + (c & 1) * S::kSum + 16 * set;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              if (16 * (2 * u + set) < part_cols) {
                float y[16];
                tmem_ld16_ahead(src + 32 * u, y);
                tmem_ld_wait(y);
#pragma unroll
                for (int n = 0; n < 16; ++n) acc[u][n] += __float2int_rn(y[n]);
              }
            }
            sum_done();
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int n = j * kI8Part + 16 * (2 * u + set);
            if (ok && 2 * j + u < kMine && n < p.cols) {
              float y[16];
#pragma unroll
              for (int m = 0; m < 16; ++m) y[m] = (float)acc[u][m];
              write(y, hs[2 * j + u < kMine ? 2 * j + u : 0], n);
            }
          }
        }
      }
    }
  }
  if (!ok) {
    report(a.err, 4u);
    let_settle();
  }
  __syncwarp();
  tmem_fence_before();
  cluster_sync_all();
  tmem_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tbase), "r"(512) : "memory");
}

template <int NT, bool kBf16>
cudaError_t launch_i8(const HeadI8Args& a, const I8Plan& p, int grid, int dev, const CUtensorMap& mw,
                      const CUtensorMap& mh, const CUtensorMap& mp, cudaStream_t s) {
  static unsigned long long done = 0ull;
  const unsigned long long bit = 1ull << (dev & 63);
  if (!(__atomic_load_n(&done, __ATOMIC_ACQUIRE) & bit)) {
    const cudaError_t e = cudaFuncSetAttribute(head_i8_kernel<NT, kBf16>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)I8Shape<NT>::kSmem);
    if (e != cudaSuccess) return e;
    __atomic_fetch_or(&done, bit, __ATOMIC_ACQ_REL);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kI8Threads);
  cfg.dynamicSmemBytes = I8Shape<NT>::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, head_i8_kernel<NT, kBf16>, a, p, mw, mh, mp);
}
template <bool kBf16>
cudaError_t launch_i8_cols(const HeadI8Args& a, const I8Plan& p, int grid, int dev, const CUtensorMap& mw,
                           const CUtensorMap& mh, const CUtensorMap& mp, cudaStream_t s) {
  if (p.cols <= 32) return launch_i8<32, kBf16>(a, p, grid, dev, mw, mh, mp, s);
  if (p.cols <= 64) return launch_i8<64, kBf16>(a, p, grid, dev, mw, mh, mp, s);
  if (p.cols <= 128) return launch_i8<128, kBf16>(a, p, grid, dev, mw, mh, mp, s);
  return launch_i8<192, kBf16>(a, p, grid, dev, mw, mh, mp, s);
}
}  // namespace

cudaError_t launch_quantize_rows(const void* x, int dtype, int R, int d, int8_t* q, float* scale, cudaStream_t s) {
  return dtype == 0 ? launch_quantize((const float*)x, R, d, q, scale, s)
                    : launch_quantize((const __nv_bfloat16*)x, R, d, q, scale, s);
}

cudaError_t take_head_i8_errors(unsigned* flags, cudaStream_t s) { return take_errors(flags, s); }

cudaError_t launch_head_i8(const HeadI8Args& a, cudaStream_t s) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  if (sms < 1) sms = 1;
  const int64_t pairs = sms / 2 > 0 ? sms / 2 : 1;
  I8Plan p;
  // Tiles of up to 192 tokens: as many accumulator columns, twice, as leave room
  // for two buffers of the turned weight (d=1024 V=32000, us against tiles of up to
  // 128: R=192 20.9, 25.0; R=384 30.9, 30.3; R=512 35.7, 37.1; R=1024 57, 62).
  p.rt = (a.R + 191) / 192;
  p.cols = ((a.R + p.rt - 1) / p.rt + 31) / 32 * 32;
  p.rt = (a.R + p.cols - 1) / p.cols;
  // one tile of tokens: the weight is streamed once, so its rows are spread
  // evenly over the SMs; more of them: whole tiles
  const int64_t wave = pairs * 2 * kI8Rows, waves = (a.V + wave - 1) / wave;
  p.height = p.rt > 1 ? kI8Rows : (int)(((a.V + 2 * pairs * waves - 1) / (2 * pairs * waves) + 3) / 4 * 4);
  p.vt = (int)((a.V + 2 * (int64_t)p.height - 1) / (2 * p.height));
  CUtensorMap mw, mh, mp;
  if (!tma_matrix(&mw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.weight, a.d, a.V, p.height) ||
      !tma_matrix(&mh, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, a.h16, a.d, a.R, p.cols / 2))
    return cudaErrorInvalidValue;
  mp = mh;                                          // (a part is the tile)
  if (p.cols > kI8Part && !tma_matrix(&mp, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, a.h16, a.d, a.R, kI8Part / 2))
    return cudaErrorInvalidValue;
  head_i8_tokens_kernel<<<a.R < 65536 ? a.R : 65536, kTokenThreads, 0, s>>>(a);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const int64_t tiles = (int64_t)p.vt * p.rt;       // (31 bits hold them: R V < 2^46, V <= 2^30)
  const int grid = (int)(2 * (tiles < pairs ? tiles : pairs));
  return a.dtype == 0 ? launch_i8_cols<false>(a, p, grid, dev, mw, mh, mp, s) : launch_i8_cols<true>(a, p, grid, dev, mw, mh, mp, s);
}

}  // namespace cmsd
