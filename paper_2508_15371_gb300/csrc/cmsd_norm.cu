// Layer norm (include/cmsd.h, cmsd_layernorm) and its gradients
// (cmsd_layernorm_backward).
//
// A row stays in the registers of its threads between its sums and what they give,
// and is read once, but for rows over 32768 columns forward (three times), gradients
// of few rows (twice) and of over 8192 columns (d_x and the sums over rows each by
// itself).  Bound by memory.
#include <cuda_bf16.h>

#include <algorithm>

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
        const float4 v = *reinterpret_cast<const float4*>(q + k);
        f[k] = v.x; f[k + 1] = v.y; f[k + 2] = v.z; f[k + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < VE; ++k) f[k] = q[k];
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + j;
    if constexpr (VE % 4 == 0) {
#pragma unroll
      for (int k = 0; k < VE; k += 4) {
        const uint2 v = *reinterpret_cast<const uint2*>(q + k);
        f[k] = bf_lo(v.x); f[k + 1] = bf_hi(v.x); f[k + 2] = bf_lo(v.y); f[k + 3] = bf_hi(v.y);
      }
    } else {
#pragma unroll
      for (int k = 0; k < VE; ++k) f[k] = __uint_as_float((uint32_t)q[k] << 16);
    }
  }
}

// the sums of N numbers over a CTA of W warps, in every thread; buf: [W][N] for each use, so that no
// two uses without a barrier between them share one
template <int N, int W>
__device__ __forceinline__ void row_sums(float (&v)[N], float* buf) {
#pragma unroll
  for (int o = 16; o; o >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(kFull, v[k], o);
  const int w = threadIdx.x >> 5;
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

// ---- numbers of a vector ------------------------------------------------------------------
// VE numbers in pairs, two an instruction, or one by one where rows begin on odd
// entries.
template <int VE>
struct Num {
  using N = u64;
  static constexpr int kN = VE / 2;
  static __device__ __forceinline__ N all(float x) { return pack2(x, x); }
  static __device__ __forceinline__ N add(N a, N b) { return add2(a, b); }
  static __device__ __forceinline__ N mul(N a, N b) { return mul2(a, b); }
  static __device__ __forceinline__ N fma(N a, N b, N c) { return fma2(a, b, c); }
  static __device__ __forceinline__ float sum(N a) { return lo32f(a) + hi32f(a); }
  static __device__ __forceinline__ N of(const float (&f)[VE], int j) { return pack2(f[2 * j], f[2 * j + 1]); }
  static __device__ __forceinline__ void to(N a, float* f) { f[0] = lo32f(a); f[1] = hi32f(a); }
  template <typename T>
  static __device__ __forceinline__ void get(const typename RowVec<T, VE>::Raw& r, N (&n)[kN]) { get_pairs<T, VE>(r, n); }
  template <typename T>
  static __device__ __forceinline__ typename RowVec<T, VE>::Raw put(const N (&n)[kN]) { return put_pairs<T, VE>(n); }
};
template <>
struct Num<1> {
  using N = float;
  static constexpr int kN = 1;
  static __device__ __forceinline__ N all(float x) { return x; }
  static __device__ __forceinline__ N add(N a, N b) { return a + b; }
  static __device__ __forceinline__ N mul(N a, N b) { return a * b; }
  static __device__ __forceinline__ N fma(N a, N b, N c) { return __fmaf_rn(a, b, c); }
  static __device__ __forceinline__ float sum(N a) { return a; }
  static __device__ __forceinline__ N of(const float (&f)[1], int) { return f[0]; }
  static __device__ __forceinline__ void to(N a, float* f) { f[0] = a; }
  template <typename T>
  static __device__ __forceinline__ void get(const typename RowVec<T, 1>::Raw& r, N (&n)[1]) { RowVec<T, 1>::get(r, n); }
  template <typename T>
  static __device__ __forceinline__ typename RowVec<T, 1>::Raw put(const N (&n)[1]) { return RowVec<T, 1>::put(n); }
};

// ---- rows on their way through shared memory ---------------------------------------------
// A row is copied as the 16-byte pieces that it touches (the last row's end alone is
// cut short), so rows that begin anywhere come as fast as aligned ones; those are
// then read by other threads than copied them, and a barrier stands between.
template <typename T, int VE>
__host__ __device__ constexpr bool aligned_rows() { return VE * sizeof(T) == 16; }
__device__ __forceinline__ void copy_async(uint32_t to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void close_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_but() {       // all but the last N groups have arrived
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// row `row` of x [R][d], if there is one, by threads t of n, kTurns pieces each (a row that begins within a piece
// may have one more)
template <typename T, int VE, int kTurns>
__device__ __forceinline__ void request_row(uint32_t to, const void* x, int row, const NormArgs& a, int t, int n) {
  if (row >= a.R) return;
  const int bytes = a.d * (int)sizeof(T);
  const char* p = static_cast<const char*>(x) + (int64_t)row * bytes;
  if constexpr (VE * sizeof(T) == 16) {
    p += t * 16;
    to += t * 16;
#pragma unroll
    for (int k = 0; k < kTurns; ++k)
      if ((t + n * k) * 16 < bytes) copy_async(to + n * k * 16, p + n * k * 16, 16);
  } else {
    const int lead = (int)(reinterpret_cast<uintptr_t>(p) & 15), last = lead + bytes;
    const int64_t rest = (int64_t)(a.R - row) * bytes + lead;          // bytes from the first piece to the end of x
    p -= lead;
#pragma unroll
    for (int k = 0; k <= kTurns; ++k) {
      const int at = (t + n * k) * 16;
      if ((k < kTurns || t == 0) && at < last) copy_async(to + at, p + at, rest - at < 16 ? (int)(rest - at) : 16);
    }
  }
}
// its vector v (VE entries); row's first byte is at `to` + lead
template <typename T, int VE>
__device__ __forceinline__ typename RowVec<T, VE>::Raw staged(const char* to, int lead, int v) {
  return *reinterpret_cast<const typename RowVec<T, VE>::Raw*>(to + lead + v * (int)(VE * sizeof(T)));
}
template <typename T, int VE>
__device__ __forceinline__ int lead_of(int row, int d) {
  return VE * sizeof(T) == 16 ? 0 : (int)((unsigned)row * (unsigned)d * (unsigned)sizeof(T) & 15u);
}

// ---- few rows, and wide ones -----------------------------------------------------------------
// A CTA of W warps a row, NV vectors of VE entries a thread.  A first mean c is that of
// the differences from the row's first entry, so that a row of one number gives
// exactly bias; it is as far off as that entry's size makes it.  Differences from c
// are of the entries themselves, and what c lacks, e, is their mean and comes with
// their squares: no entry loses bits to another one, wherever a large one stands.
template <typename T, int VE, int NV, int W>
__global__ void __launch_bounds__(32 * W) norm_kernel(const NormArgs a) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
  using M = Num<VE>;
  using N = typename M::N;
  constexpr int kN = M::kN;
  __shared__ float s_sum[3 * W];
  wait_for_previous();
  const int nvec = a.d / VE, t = threadIdx.x;
  const int64_t row = blockIdx.x;
  const Raw* x = static_cast<const Raw*>(a.x) + (size_t)row * nvec;
  Raw* y = static_cast<Raw*>(a.y) + (size_t)row * nvec;
  Raw raw[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    raw[k] = V::zero();
    if (t + 32 * W * k < nvec) raw[k] = __ldcs(x + t + 32 * W * k);
  }
  const float pilot = to_float(static_cast<const T*>(a.x)[(size_t)row * a.d]);
  // few entries a thread: the parameters' too are requested before the sums
  constexpr bool kEarly = VE * NV <= 16;
  float w[kEarly ? NV : 1][VE], b[kEarly ? NV : 1][VE];
  const auto parameters = [&](int k, int v) {
    if (a.weight) params<VE>(a.weight, a.wdtype, v * VE, w[k]);
    if (a.bias) params<VE>(a.bias, a.wdtype, v * VE, b[k]);
  };
  if constexpr (kEarly) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (t + 32 * W * k < nvec) parameters(k, t + 32 * W * k);
  }
  N h[NV][kN], n1 = M::all(0.f), n2 = M::all(0.f), p = M::all(-pilot);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    M::template get<T>(raw[k], h[k]);
    if (t + 32 * W * k < nvec)
#pragma unroll
      for (int j = 0; j < kN; ++j) n1 = M::add(n1, M::add(h[k][j], p));
  }
  float s[1] = {M::sum(n1)};
  row_sums<1, W>(s, s_sum);
  const float c = pilot + s[0] / a.d;
  p = M::all(-c);
  n1 = M::all(0.f);
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (t + 32 * W * k < nvec)
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        h[k][j] = M::add(h[k][j], p);
        n1 = M::add(n1, h[k][j]);
        n2 = M::fma(h[k][j], h[k][j], n2);
      }
  float q[2] = {M::sum(n1), M::sum(n2)};
  row_sums<2, W>(q, s_sum + W);
  const float e = q[0] / a.d, rstd = 1.f / sqrtf((q[1] / a.d - e * e) + a.eps);
  if (t == 0) {
    if (a.mean) a.mean[row] = c + e;
    if (a.rstd) a.rstd[row] = rstd;
  }
  const N scale = M::all(rstd), shift = M::all(-e * rstd);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = t + 32 * W * k;
    if (v >= nvec) continue;
    const int q = kEarly ? k : 0;
    if (!kEarly) parameters(q, v);
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      h[k][j] = M::fma(h[k][j], scale, shift);
      if (a.weight && a.bias) h[k][j] = M::fma(h[k][j], M::of(w[q], j), M::of(b[q], j));
      else if (a.weight) h[k][j] = M::mul(h[k][j], M::of(w[q], j));
      else if (a.bias) h[k][j] = M::add(h[k][j], M::of(b[q], j));
    }
    y[v] = M::template put<T>(h[k]);
  }
}

// rows of over 32768 entries, which do not fit: a CTA a row, read three times (from L2)
constexpr int kWide = 1024;
template <typename T>
__global__ void __launch_bounds__(kWide) norm_wide_kernel(const NormArgs a) {
  __shared__ float s_sum[3 * kWide / 32];
  wait_for_previous();
  const T* x = static_cast<const T*>(a.x) + (size_t)blockIdx.x * a.d;
  T* y = static_cast<T*>(a.y) + (size_t)blockIdx.x * a.d;
  const float pilot = to_float(x[0]);
  float s[1] = {0.f};
  for (int j = threadIdx.x; j < a.d; j += kWide) s[0] += to_float(x[j]) - pilot;
  row_sums<1, kWide / 32>(s, s_sum);
  const float c = pilot + s[0] / a.d;
  float q[2] = {0.f, 0.f};
  for (int j = threadIdx.x; j < a.d; j += kWide) {
    const float h = to_float(x[j]) - c;
    q[0] += h;
    q[1] = __fmaf_rn(h, h, q[1]);
  }
  row_sums<2, kWide / 32>(q, s_sum + kWide / 32);
  const float e = q[0] / a.d, rstd = 1.f / sqrtf((q[1] / a.d - e * e) + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[blockIdx.x] = c + e;
    if (a.rstd) a.rstd[blockIdx.x] = rstd;
  }
  for (int j = threadIdx.x; j < a.d; j += kWide) {
    float h = ((to_float(x[j]) - c) - e) * rstd;
    if (a.weight) h *= param(a.weight, a.wdtype, j);
    if (a.bias) h += param(a.bias, a.wdtype, j);
    y[j] = from_float<T>(h);
  }
}

// ---- many rows -----------------------------------------------------------------------------
// A grid that stays: a thread has the same columns in all of its rows, with their
// parameters (forward) or their sums over rows (gradients) in registers; W warps a
// row, kGroups rows of a CTA at a time.  Rows come through a ring in shared
// memory.  Bound by memory forward (R = 16384 d = 2048 bf16 22.7 us, 5.9 TB/s), by
// memory and a barrier a row backward (36.6 us with the join, 5.5 TB/s).  Sixteen
// columns a thread: of eight, exchanging a row's sums is most of the work (46 us
// forward); with a warp a row the parameters are read again for every row (34 us).
// Forward, bf16 rows of over 256 entries take the first mean c (see norm_kernel) from
// the threads' first eight columns alone, which every row fills: a power of two of
// entries added in pairs, so that of equal ones it is exact.  It is off by at most s,
// the mean of |x - mean|, beside its rounding, which is far below a bf16 entry's: the
// mean of squares that e's square is taken from is not above var + s^2 <= 2 var.  From
// all columns 0.6 us more.  f32 rows, whose last bits a sum of entries would touch, have
// their bytes to wait for: 22.5 us either way (R = 8192 d = 2048).
constexpr int kSms = 152;
__host__ __device__ constexpr int cta_threads(int w) { return w > 8 ? 32 * w : 256; }
__host__ __device__ constexpr int cta_groups(int w) { return cta_threads(w) / (32 * w); }
__host__ __device__ constexpr int staged_bytes(int w, int cols, int size) { return 32 * w * cols * size + 16; }     // of a row
// a barrier of the W warps of a row (the CTA's groups go their own ways)
template <int W>
__device__ __forceinline__ void group_sync(int group) {
  if (W == 1) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(32 * W) : "memory");
}
// the sum of W numbers in shared memory
template <int W>
__device__ __forceinline__ float sum_of(const float* buf) {
  float v = 0.f;
  if constexpr (W % 4 == 0) {
#pragma unroll
    for (int j = 0; j < W; j += 4) {
      const float4 p = *reinterpret_cast<const float4*>(buf + j);
      v += (p.x + p.y) + (p.z + p.w);
    }
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) v += buf[j];
  }
  return v;
}
// the sums of N numbers over a group's warps, in every thread; buf: [N][W], not in use by another exchange between
// whose barrier and this one's there is none
template <int N, int W>
__device__ __forceinline__ void group_sums(float (&v)[N], float* buf, int group) {
#pragma unroll
  for (int o = 16; o; o >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(kFull, v[k], o);
  if (W == 1) return;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) buf[k * W + (threadIdx.x >> 5) % W] = v[k];
  group_sync<W>(group);
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = sum_of<W>(buf + k * W);
}

// The same of two numbers: from the first exchange on, half of the lanes have one and half the other.
template <int W>
__device__ __forceinline__ void group_two_sums(float (&v)[2], float* buf, int group) {
  const int lane = threadIdx.x & 31;
  const bool second = (lane & 16) != 0;
  const float gives = second ? v[0] : v[1], keeps = second ? v[1] : v[0];
  float x = keeps + __shfl_xor_sync(kFull, gives, 16);
#pragma unroll
  for (int o = 8; o; o >>= 1) x += __shfl_xor_sync(kFull, x, o);
  if (W == 1) {
    v[0] = __shfl_sync(kFull, x, 0);
    v[1] = __shfl_sync(kFull, x, 16);
    return;
  }
  if ((lane & 15) == 0) buf[(lane >> 4) * W + (threadIdx.x >> 5) % W] = x;
  group_sync<W>(group);
#pragma unroll
  for (int k = 0; k < 2; ++k) v[k] = sum_of<W>(buf + k * W);
}

// v^(-1/2): one Newton step behind CUDA's, to 2 u.  (With 1 / sqrtf, whose steps wait for one another, R = 16384
// d = 2048 bf16 took 23.3 us forward instead of 22.6, d = 256 8.5 instead of 7.9.)
__device__ __forceinline__ float inverse_root(float v) {
  const float near = rsqrtf(v);
  return __fmaf_rn(near * 0.5f, __fmaf_rn(-near * v, near, 1.f), near);
}

// whether a thread's vector k is in the row: a row that takes W > 1 warps fills half of what they hold
template <int W, int NV>
__device__ __forceinline__ bool in_row(int t, int k, int nvec) {
  return (W > 1 && 2 * (k + 1) <= NV) || t + 32 * W * k < nvec;
}

constexpr int kNormStages = 3;
__host__ __device__ constexpr int norm_ctas(int cols) { return cols > 8 ? 3 : 4; }             // an SM, by registers
template <typename T, int VE, int kCols, int W>
__global__ void __launch_bounds__(cta_threads(W), norm_ctas(kCols)) norm_many_kernel(const NormArgs a) {
  using Raw = typename RowVec<T, VE>::Raw;
  using M = Num<VE>;
  using N = typename M::N;
  constexpr int kN = M::kN, NV = kCols / VE, kGroups = cta_groups(W);
  constexpr int kRowBytes = staged_bytes(W, kCols, sizeof(T)), kTurns = kCols * sizeof(T) / 16;
  // vectors of a thread that every row fills (W = 1: rows of over 256) and that c is made from, or 0: from all
  constexpr int kHalf = sizeof(T) == 2 && kCols > 8 ? NV / 2 : 0;
  extern __shared__ uint4 s_ring4[];
  __shared__ __align__(16) float s_sum[W > 1 ? 3 * kGroups * W : 1];
  wait_for_previous();
  const int nvec = a.d / VE, t = threadIdx.x % (32 * W), group = threadIdx.x / (32 * W);
  const int64_t first = (int64_t)blockIdx.x * kGroups + group, step = (int64_t)gridDim.x * kGroups;
  char* ring = reinterpret_cast<char*>(s_ring4) + group * kNormStages * kRowBytes;       // [kNormStages]
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
  float* sums = s_sum + (W > 1 ? 3 * group * W : 0);
  const auto request = [&](int64_t row, int stage) {
    request_row<T, VE, kTurns>(ring_at + stage * kRowBytes, a.x, row, a, t, 32 * W);
    close_copies();
  };
#pragma unroll
  for (int k = 0; k < kNormStages - 1; ++k) request(first + k * step, k);
  N w[NV][kN], b[NV][kN];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float f[VE], h[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      f[j] = 1.f;
      h[j] = 0.f;
    }
    if (in_row<W, NV>(t, k, nvec)) {
      if (a.weight) params<VE>(a.weight, a.wdtype, (t + 32 * W * k) * VE, f);
      if (a.bias) params<VE>(a.bias, a.wdtype, (t + 32 * W * k) * VE, h);
    }
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      w[k][j] = M::of(f, j);
      b[k][j] = M::of(h, j);
    }
  }
  const float over_d = 1.f / a.d;
  int stage = 0;
  for (int64_t row = first; row < a.R; row += step) {
    copies_but<kNormStages - 2>();
    group_sync<W>(group);                             // (the first entry is another thread's copy, if no more is)
    request(row + (kNormStages - 1) * step, stage == 0 ? kNormStages - 1 : stage - 1);
    const char* from = ring + stage * kRowBytes;
    const int lead = lead_of<T, VE>(row, a.d);
    N h[NV][kN];
    float s[1], c;
    if constexpr (kHalf > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (in_row<W, NV>(t, k, nvec)) M::template get<T>(staged<T, VE>(from, lead, t + 32 * W * k), h[k]);
      N v[kHalf * kN];
#pragma unroll
      for (int j = 0; j < kHalf * kN; ++j) v[j] = h[j / kN][j % kN];
#pragma unroll
      for (int o = kHalf * kN / 2; o; o >>= 1)
#pragma unroll
        for (int j = 0; j < o; ++j) v[j] = M::add(v[j], v[j + o]);
      s[0] = M::sum(v[0]);
      group_sums<1, W>(s, sums, group);
      c = s[0] * (1.f / (32 * W * kHalf * VE));
    } else {
      const float first_entry = to_float(*reinterpret_cast<const T*>(from + lead));
      N sum = M::all(0.f);
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (in_row<W, NV>(t, k, nvec)) {
          M::template get<T>(staged<T, VE>(from, lead, t + 32 * W * k), h[k]);
#pragma unroll
          for (int j = 0; j < kN; ++j) sum = M::add(sum, M::add(h[k][j], M::all(-first_entry)));
        }
      s[0] = M::sum(sum);
      group_sums<1, W>(s, sums, group);
      c = __fmaf_rn(s[0], over_d, first_entry);
    }
    stage = stage + 1 == kNormStages ? 0 : stage + 1;
    const N p = M::all(-c);
    N n1 = M::all(0.f), n2 = M::all(0.f);
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (in_row<W, NV>(t, k, nvec))
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          h[k][j] = M::add(h[k][j], p);
          n1 = M::add(n1, h[k][j]);
          n2 = M::fma(h[k][j], h[k][j], n2);
        }
    float q[2] = {M::sum(n1), M::sum(n2)};
    if (W == 1) group_sums<2, W>(q, sums + W, group);   // (every lane has both at once: d = 512 4.84 us, not 4.94)
    else group_two_sums<W>(q, sums + W, group);
    const float e = q[0] * over_d, rstd = inverse_root(__fmaf_rn(-e, e, __fmaf_rn(q[1], over_d, a.eps)));
    if (t == 0) {
      if (a.mean) a.mean[row] = c + e;
      if (a.rstd) a.rstd[row] = rstd;
    }
    const N scale = M::all(rstd), shift = M::all(-e * rstd);
    Raw* y = static_cast<Raw*>(a.y) + (size_t)row * nvec;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (in_row<W, NV>(t, k, nvec)) {
#pragma unroll
        for (int j = 0; j < kN; ++j) h[k][j] = M::fma(M::fma(h[k][j], scale, shift), w[k][j], b[k][j]);
        y[t + 32 * W * k] = M::template put<T>(h[k]);
      }
  }
  copies_but<0>();
}

// ---- gradients ---------------------------------------------------------------------------
// The CTAs' sums over rows are joined by norm_join_kernel, in the order of the CTAs.
__host__ __device__ constexpr int grad_stages(int size) { return size == 2 ? 3 : 2; }
__host__ __device__ constexpr int grad_smem(int w, int cols, int size) {
  return grad_stages(size) * 2 * cta_groups(w) * staged_bytes(w, cols, size);
}
__host__ __device__ constexpr int grad_ctas(int w, int cols) { return w > 8 ? 1 : (cols > 8 ? 2 : 3); }       // an SM, by registers
template <typename T, int VE, int kCols, int W>
__global__ void __launch_bounds__(cta_threads(W), grad_ctas(W, kCols)) norm_backward_kernel(const NormArgs a) {
  using Raw = typename RowVec<T, VE>::Raw;
  using M = Num<VE>;
  using N = typename M::N;
  constexpr int kN = M::kN, NV = kCols / VE, kGroups = cta_groups(W), kThreads = cta_threads(W);
  constexpr int kStages = grad_stages(sizeof(T)), kRowBytes = staged_bytes(W, kCols, sizeof(T)), kTurns = kCols * sizeof(T) / 16;
  extern __shared__ uint4 s_ring4[];
  __shared__ __align__(16) float s_sum[W > 1 ? 2 * kGroups * 2 * W : 1];
  wait_for_previous();
  const int nvec = a.d / VE, t = threadIdx.x % (32 * W), group = threadIdx.x / (32 * W);
  const int first = blockIdx.x * kGroups + group, step = gridDim.x * kGroups;
  char* ring = reinterpret_cast<char*>(s_ring4) + group * kStages * 2 * kRowBytes;             // [kStages][2]
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
  const auto request = [&](int row, int stage) {
    const uint32_t to = ring_at + stage * 2 * kRowBytes;
    request_row<T, VE, kTurns>(to, a.x, row, a, t, 32 * W);
    request_row<T, VE, kTurns>(to + kRowBytes, a.d_y, row, a, t, 32 * W);
    close_copies();
  };
#pragma unroll
  for (int k = 0; k < kStages - 1; ++k) request(first + k * step, k);
  float mean = first < a.R ? a.mean_in[first] : 0.f, rstd = first < a.R ? a.rstd_in[first] : 0.f;
  N w[NV][kN], dw[NV][kN], db[NV][kN];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float f[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = 1.f;
    if (a.weight && in_row<W, NV>(t, k, nvec)) params<VE>(a.weight, a.wdtype, (t + 32 * W * k) * VE, f);
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      w[k][j] = M::of(f, j);
      dw[k][j] = db[k][j] = M::all(0.f);
    }
  }
  const float over_d = 1.f / a.d;
  int stage = 0, turn = 0;
  for (int row = first; row < a.R; row += step, turn ^= 1) {
    copies_but<kStages - 2>();
    if (!aligned_rows<T, VE>()) group_sync<W>(group);
    request(row + (kStages - 1) * step, stage == 0 ? kStages - 1 : stage - 1);
    const char* from = ring + stage * 2 * kRowBytes;
    const int lead = lead_of<T, VE>(row, a.d);
    stage = stage + 1 == kStages ? 0 : stage + 1;
    const float r = rstd;
    const N m = M::all(-mean), rs = M::all(r);
    if (row + step < a.R) {
      mean = a.mean_in[row + step];
      rstd = a.rstd_in[row + step];
    }
    N h[NV][kN], g[NV][kN], s1 = M::all(0.f), s2 = M::all(0.f);
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (in_row<W, NV>(t, k, nvec)) {
        M::template get<T>(staged<T, VE>(from, lead, t + 32 * W * k), h[k]);
        M::template get<T>(staged<T, VE>(from + kRowBytes, lead, t + 32 * W * k), g[k]);
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          h[k][j] = M::mul(M::add(h[k][j], m), rs);
          dw[k][j] = M::fma(g[k][j], h[k][j], dw[k][j]);
          db[k][j] = M::add(db[k][j], g[k][j]);
          g[k][j] = M::mul(g[k][j], w[k][j]);
          s1 = M::add(s1, g[k][j]);
          s2 = M::fma(g[k][j], h[k][j], s2);
        }
      }
    if (!a.d_x) continue;                             // (the same in the whole grid)
    float s[2] = {M::sum(s1), M::sum(s2)};
    group_two_sums<W>(s, s_sum + (W > 1 ? (turn * kGroups + group) * 2 * W : 0), group);
    const N m1 = M::all(-s[0] * over_d * r), m2 = M::all(-s[1] * over_d * r);
    Raw* d_x = static_cast<Raw*>(a.d_x) + (size_t)row * nvec;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (in_row<W, NV>(t, k, nvec)) {
#pragma unroll
        for (int j = 0; j < kN; ++j) g[k][j] = M::fma(h[k][j], m2, M::fma(g[k][j], rs, m1));
        d_x[t + 32 * W * k] = M::template put<T>(g[k]);
      }
  }
  copies_but<0>();
  if (!a.d_weight && !a.d_bias) return;
  // the groups' sums, in their order, through the ring's memory
  float* s_col = reinterpret_cast<float*>(s_ring4);
  float* part = a.part + (size_t)blockIdx.x * 2 * a.d;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float sum[NV][VE];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < kN; ++j) M::to(which ? db[k][j] : dw[k][j], &sum[k][VE / kN * j]);
    if (kGroups > 1) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < VE; ++j) s_col[(k * VE + j) * kThreads + threadIdx.x] = sum[k][j];
      __syncthreads();
    }
    if (group == 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (in_row<W, NV>(t, k, nvec)) {
#pragma unroll
          for (int j = 0; j < VE; ++j)
            for (int q = 1; q < kGroups; ++q) sum[k][j] += s_col[(k * VE + j) * kThreads + 32 * W * q + t];
          float* p = part + which * a.d + (t + 32 * W * k) * VE;
          // (one by one, each goes to a sector of its own: R = 4096 d = 2048 17.4 us instead of 14.3)
          if constexpr (VE % 4 == 0) {
#pragma unroll
            for (int j = 0; j < VE; j += 4)
              *reinterpret_cast<float4*>(p + j) = make_float4(sum[k][j], sum[k][j + 1], sum[k][j + 2], sum[k][j + 3]);
          } else if constexpr (VE == 2) {
            *reinterpret_cast<float2*>(p) = make_float2(sum[k][0], sum[k][1]);
          } else {
            *p = sum[k][0];
          }
        }
    }
  }
}

// a CTA 32 columns of one of the two, each of its warps a part of the CTAs' sums
// (eight warps or 32 by the parts: 32 of few parts, 1024 x 16384 f32, 8 us more)
constexpr int kJoinAhead = 10;                       // parts of a warp requested at once
template <int kJoinWarps>
__global__ void __launch_bounds__(32 * kJoinWarps) norm_join_kernel(const NormArgs a, int parts) {
  __shared__ float s_part[kJoinWarps][32];
  const int lane = threadIdx.x & 31, j = blockIdx.x * 32 + lane, which = blockIdx.y, warp = threadIdx.x >> 5;
  void* out = which ? a.d_bias : a.d_weight;
  wait_for_previous();
  if (!out) return;
  float v = 0.f;
  if (j < a.d)
    for (int p0 = warp; p0 < parts; p0 += kJoinWarps * kJoinAhead) {
      float x[kJoinAhead];
#pragma unroll
      for (int u = 0; u < kJoinAhead; ++u) {
        const int p = p0 + u * kJoinWarps;
        x[u] = p < parts ? __ldcg(a.part + ((size_t)p * 2 + which) * a.d + j) : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kJoinAhead; ++u) v += x[u];
    }
  s_part[warp][lane] = v;
  __syncthreads();
  if (warp || j >= a.d) return;
  float sum[kJoinWarps];                             // in pairs: one after another is 1.4e-7 off, not 0.9e-7, at R = 333
#pragma unroll
  for (int k = 0; k < kJoinWarps; ++k) sum[k] = s_part[k][lane];
#pragma unroll
  for (int o = kJoinWarps / 2; o; o >>= 1)
#pragma unroll
    for (int k = 0; k < o; ++k) sum[k] += sum[k + o];
  v = sum[0];
  if (a.wdtype == 0) static_cast<float*>(out)[j] = v;
  else static_cast<__nv_bfloat16*>(out)[j] = __float2bfloat16_rn(v);
}

// ---- gradients of few rows ---------------------------------------------------------------
// One launch, nothing joined: the first `cols` CTAs have kFewCols vectors of columns
// each and all rows' sums of them (32 rows at once, eight of a thread requested
// together), the others a row of d_x each.  Inputs are read twice, the second time
// from L2; a few loads in a row bound it.
constexpr int kFewCols = 8, kFewLanes = 32, kFewThreads = kFewCols * kFewLanes, kFewAhead = 8;
template <typename T, int VE, int NV>
__global__ void __launch_bounds__(kFewThreads) norm_backward_few_kernel(const NormArgs a, int cols) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
  using M = Num<VE>;
  using N = typename M::N;
  constexpr int kN = M::kN, W = kFewThreads / 32;
  __shared__ float s_sum[2 * W];
  __shared__ float s_col[2][kFewLanes][kFewCols * VE + 1];
  wait_for_previous();
  const int nvec = a.d / VE, t = threadIdx.x;
  const Raw* xs = static_cast<const Raw*>(a.x);
  const Raw* gs = static_cast<const Raw*>(a.d_y);
  if ((int)blockIdx.x < cols) {
    const int v = blockIdx.x * kFewCols + t % kFewCols, lane = t / kFewCols;
    N w[kN], b[kN];
#pragma unroll
    for (int j = 0; j < kN; ++j) w[j] = b[j] = M::all(0.f);
    if (v < nvec)
#pragma unroll 1
      for (int r0 = lane; r0 < a.R; r0 += kFewLanes * kFewAhead) {
        Raw x[kFewAhead], y[kFewAhead];
        float mean[kFewAhead], rstd[kFewAhead];
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) {
          const int r = r0 + u * kFewLanes;
          x[u] = y[u] = V::zero();
          mean[u] = rstd[u] = 0.f;
          if (r < a.R) {
            x[u] = xs[(size_t)r * nvec + v];
            y[u] = gs[(size_t)r * nvec + v];
            mean[u] = a.mean_in[r];
            rstd[u] = a.rstd_in[r];
          }
        }
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) {
          N h[kN], g[kN];
          M::template get<T>(x[u], h);
          M::template get<T>(y[u], g);
          const N m = M::all(-mean[u]), rs = M::all(rstd[u]);
#pragma unroll
          for (int j = 0; j < kN; ++j) {
            w[j] = M::fma(g[j], M::mul(M::add(h[j], m), rs), w[j]);
            b[j] = M::add(b[j], g[j]);
          }
        }
      }
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      M::to(w[j], &s_col[0][lane][t % kFewCols * VE + VE / kN * j]);
      M::to(b[j], &s_col[1][lane][t % kFewCols * VE + VE / kN * j]);
    }
    __syncthreads();
    const int which = t / (kFewCols * VE), c = t % (kFewCols * VE), j = blockIdx.x * (kFewCols * VE) + c;
    void* out = which ? a.d_bias : a.d_weight;
    if (which > 1 || j >= a.d || !out) return;
    float sum[kFewLanes];                            // in pairs, as norm_join_kernel
#pragma unroll
    for (int k = 0; k < kFewLanes; ++k) sum[k] = s_col[which][k][c];
#pragma unroll
    for (int o = kFewLanes / 2; o; o >>= 1)
#pragma unroll
      for (int k = 0; k < o; ++k) sum[k] += sum[k + o];
    if (a.wdtype == 0) static_cast<float*>(out)[j] = sum[0];
    else static_cast<__nv_bfloat16*>(out)[j] = __float2bfloat16_rn(sum[0]);
    return;
  }
  const int row = blockIdx.x - cols;
  xs += (size_t)row * nvec;
  gs += (size_t)row * nvec;
  Raw x[NV], y[NV];
  float w[NV][VE];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = t + kFewThreads * k;
    x[k] = y[k] = V::zero();
#pragma unroll
    for (int j = 0; j < VE; ++j) w[k][j] = 1.f;
    if (v < nvec) {
      x[k] = xs[v];
      y[k] = gs[v];
      if (a.weight) params<VE>(a.weight, a.wdtype, v * VE, w[k]);
    }
  }
  const float r = a.rstd_in[row], over_d = 1.f / a.d;
  const N m = M::all(-a.mean_in[row]), rs = M::all(r);
  N h[NV][kN], g[NV][kN], s1 = M::all(0.f), s2 = M::all(0.f);
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (t + kFewThreads * k < nvec) {
      M::template get<T>(x[k], h[k]);
      M::template get<T>(y[k], g[k]);
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        h[k][j] = M::mul(M::add(h[k][j], m), rs);
        g[k][j] = M::mul(g[k][j], M::of(w[k], j));
        s1 = M::add(s1, g[k][j]);
        s2 = M::fma(g[k][j], h[k][j], s2);
      }
    }
  float s[2] = {M::sum(s1), M::sum(s2)};
  row_sums<2, W>(s, s_sum);
  const N m1 = M::all(-s[0] * over_d * r), m2 = M::all(-s[1] * over_d * r);
  Raw* d_x = static_cast<Raw*>(a.d_x) + (size_t)row * nvec;
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (t + kFewThreads * k < nvec) {
#pragma unroll
      for (int j = 0; j < kN; ++j) g[k][j] = M::fma(h[k][j], m2, M::fma(g[k][j], rs, m1));
      d_x[t + kFewThreads * k] = M::template put<T>(g[k]);
    }
}

constexpr int kWideCols = 8192;
// rows of over kWideCols columns: d_x by a CTA a row, the sums over rows by a CTA 32 vectors of columns; both read
// both inputs (R = 2048 d = 16384 bf16 92 us, 2.2 TB/s of what is needed)
constexpr int kWideDx = 512;                          // (two rows an SM: with 1024 threads 106 us where this takes 92)
template <typename T, int VE>
__global__ void __launch_bounds__(kWideDx, 2) norm_wide_dx_kernel(const NormArgs a) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
  constexpr int kKept = 4;                            // a thread's first vectors stay in registers
  __shared__ float s_sum[2 * kWideDx / 32];
  wait_for_previous();
  const int nvec = a.d / VE;
  const size_t at = (size_t)blockIdx.x * nvec;
  const Raw* xs = static_cast<const Raw*>(a.x) + at;
  const Raw* gs = static_cast<const Raw*>(a.d_y) + at;
  const float mean = a.mean_in[blockIdx.x], rstd = a.rstd_in[blockIdx.x], over_d = 1.f / a.d;
  const auto values = [&](int v, const Raw& x, const Raw& y, float (&h)[VE], float (&g)[VE]) {
    float w[VE];
    V::get(x, h);
    V::get(y, g);
    if (a.weight) params<VE>(a.weight, a.wdtype, v * VE, w);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      h[j] = (h[j] - mean) * rstd;
      if (a.weight) g[j] *= w[j];
    }
  };
  float s[2] = {0.f, 0.f};
  const auto add = [&](int v, const Raw& x, const Raw& y) {
    float h[VE], g[VE];
    values(v, x, y, h, g);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      s[0] += g[j];
      s[1] = __fmaf_rn(g[j], h[j], s[1]);
    }
  };
  Raw x[kKept], y[kKept];
#pragma unroll
  for (int k = 0; k < kKept; ++k) {
    const int v = threadIdx.x + kWideDx * k;
    x[k] = y[k] = V::zero();
    if (v < nvec) {
      x[k] = xs[v];
      y[k] = gs[v];
    }
  }
#pragma unroll
  for (int k = 0; k < kKept; ++k)
    if ((int)threadIdx.x + kWideDx * k < nvec) add(threadIdx.x + kWideDx * k, x[k], y[k]);
#pragma unroll 2
  for (int v = threadIdx.x + kWideDx * kKept; v < nvec; v += kWideDx) add(v, xs[v], gs[v]);
  row_sums<2, kWideDx / 32>(s, s_sum);
  const float m1 = s[0] * over_d, m2 = s[1] * over_d;
  const auto result = [&](int v, const Raw& x, const Raw& y) {
    float h[VE], g[VE];
    values(v, x, y, h, g);
#pragma unroll
    for (int j = 0; j < VE; ++j) g[j] = rstd * ((g[j] - m1) - h[j] * m2);
    return V::put(g);
  };
  Raw* d_x = static_cast<Raw*>(a.d_x) + at;
#pragma unroll
  for (int k = 0; k < kKept; ++k)
    if ((int)threadIdx.x + kWideDx * k < nvec) x[k] = result(threadIdx.x + kWideDx * k, x[k], y[k]);
#pragma unroll
  for (int k = 0; k < kKept; ++k)                     // (apart: no weight's load waits for a store)
    if ((int)threadIdx.x + kWideDx * k < nvec) d_x[threadIdx.x + kWideDx * k] = x[k];
  for (int v = threadIdx.x + kWideDx * kKept; v < nvec; v += kWideDx) d_x[v] = result(v, xs[v], gs[v]);     // (again, from L2)
}
template <typename T, int VE>
__global__ void __launch_bounds__(256) norm_wide_sums_kernel(const NormArgs a) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
  __shared__ float s_w[8][32 * VE], s_b[8][32 * VE];
  wait_for_previous();
  const int nvec = a.d / VE, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, v = blockIdx.x * 32 + lane;
  float w[VE], b[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) w[j] = b[j] = 0.f;
  if (v < nvec)
#pragma unroll 4
    for (int64_t r = (int64_t)blockIdx.y * 8 + warp; r < a.R; r += (int64_t)gridDim.y * 8) {
      const float mean = a.mean_in[r], rstd = a.rstd_in[r];
      float x[VE], g[VE];
      V::get(static_cast<const Raw*>(a.x)[(size_t)r * nvec + v], x);
      V::get(static_cast<const Raw*>(a.d_y)[(size_t)r * nvec + v], g);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        w[j] = __fmaf_rn(g[j], (x[j] - mean) * rstd, w[j]);
        b[j] += g[j];
      }
    }
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    s_w[warp][lane * VE + j] = w[j];
    s_b[warp][lane * VE + j] = b[j];
  }
  __syncthreads();
  float* part = a.part + (size_t)blockIdx.y * 2 * a.d;
  for (int k = threadIdx.x; k < 32 * VE; k += 256) {
    const int j = blockIdx.x * 32 * VE + k;
    if (j >= a.d) break;
    float sw = 0.f, sb = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      sw += s_w[q][k];
      sb += s_b[q][k];
    }
    part[j] = sw;
    part[a.d + j] = sb;
  }
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
// columns of a thread, and warps of a row
int row_cols(int d) { return d <= 256 ? 8 : 16; }
int row_warps(int d) {
  int w = 1;
  while (w * 32 * row_cols(d) < d) w *= 2;
  return w;
}
// CTAs whose sums over rows are joined, by R and d alone
int part_count(int R, int d) {
  if (d > kWideCols) return R < 64 * 8 ? ceil_div(R, 8) : 64;
  const int w = row_warps(d), n = ceil_div(R, cta_groups(w));
  return std::min(n, kSms * grad_ctas(w, row_cols(d)));
}

// Up to this many rows of 257 to 2048 entries a CTA a row, else the grid that stays: bf16 R = 16 d = 1024 1.8 against 2.0
// us, d = 2048 R = 304 2.2 and 2.1, 608 3.1 and 3.2, 1216 4.8 and 4.1; f32 d = 2048 R = 608 3.0 and 3.3, 1216 4.6 and
// 4.6.  Up to 1024 entries the grid is ahead from some 305 rows on (d = 1001 R = 304 2.05 and 2.05, 608 2.7 and 2.1).
// Narrower and wider rows go to the grid always (R = 16 d = 256 1.8 against 1.5, d = 4096 2.3 against 2.0, R = 608 3.7 and 4.1).
constexpr int kFewRows = 608;
// Whether the gradients are norm_backward_few_kernel's, else the grid's that stays and its join.  bf16: R = 16 d = 1024 1.5
// against 3.8 us, R = 333 d = 1001 3.8 and 4.8, R = 608 d = 64 3.7 and 3.7, d = 2048 4.4 and 6.0, d = 8192 8.6 and 14.9,
// R = 900 d = 64 4.7 and 3.9, R = 1216 d = 1001 7.6 and 6.0.  Over 2048 columns, rows of multiples of four, in pairs for
// bf16: d = 2052 R = 608 5.7 and 6.0, d = 8188 13.7 and 14.8 (R = 760 6.9 and 7.8, 16.2 and 16.4); d = 4096 f32 8.1 and
// 10.5.  Others are one entry at a time for f32, for bf16 where odd: d = 2049 R = 304 6.3 and 5.7, R = 608 10.1 and 6.6;
// d = 4097 R = 152 6.9 and 6.5; f32 d = 4097 R = 304 8.1 and 8.5, R = 608 15.2 and 12.3.  Even ones of bf16 stay with
// them, since the order of the sums is the same for both types: d = 4098 R = 608 7.6 and 9.2.
bool few_gradients(int R, int d) { return d <= kWideCols && R <= (d <= 2048 || d % 4 == 0 ? 608 : 304); }
template <typename T, int VE, int kCols, int W>
cudaError_t launch_many(const NormArgs& a, cudaStream_t s) {
  constexpr int smem = kNormStages * cta_groups(W) * staged_bytes(W, kCols, sizeof(T));
  const auto kernel = norm_many_kernel<T, VE, kCols, W>;
  static unsigned long long done = 0ull;
  const cudaError_t e = allow_smem(kernel, smem, &done);
  if (e != cudaSuccess) return e;
  return launch(true, kernel, std::min(ceil_div(a.R, cta_groups(W)), kSms * norm_ctas(kCols)), cta_threads(W), smem, s, a);
}
template <typename T, int VE>
cudaError_t launch_rows(const NormArgs& a, cudaStream_t s) {
  const auto few = [&](auto kernel, int threads) { return launch(true, kernel, a.R, threads, 0, s, a); };   // a CTA a row
  if (a.d <= 4096 && (a.R > kFewRows || a.d <= 256 || a.d > 2048)) switch (row_warps(a.d)) {
      case 1: return a.d <= 256 ? launch_many<T, VE, 8, 1>(a, s) : launch_many<T, VE, 16, 1>(a, s);
      case 2: return launch_many<T, VE, 16, 2>(a, s);
      case 4: return launch_many<T, VE, 16, 4>(a, s);
      default: return launch_many<T, VE, 16, 8>(a, s);
    }
  if (a.d <= 2048) return few(norm_kernel<T, VE, 8 / VE, 8>, 256);
  if (a.d <= 8192) return few(norm_kernel<T, VE, 32 / VE, 8>, 256);
  if (a.d <= 16384) return few(norm_kernel<T, VE, 32 / VE, 16>, 512);
  if (a.d <= 32768) return few(norm_kernel<T, VE, 32 / VE, 32>, 1024);
  return few(norm_wide_kernel<T>, kWide);
}

template <typename T, int VE, int kCols, int W>
cudaError_t launch_gradients(const NormArgs& a, int parts, cudaStream_t s) {
  constexpr int smem = grad_smem(W, kCols, sizeof(T));
  static_assert(smem >= kCols * 4 * cta_threads(W) || W > 8, "the groups' sums pass through the ring");
  const auto kernel = norm_backward_kernel<T, VE, kCols, W>;
  static unsigned long long done = 0ull;
  const cudaError_t e = allow_smem(kernel, smem, &done);
  if (e != cudaSuccess) return e;
  return launch(true, kernel, parts, cta_threads(W), smem, s, a);
}
template <typename T, int VE>
cudaError_t launch_gradients(const NormArgs& a, int parts, cudaStream_t s) {
  switch (row_warps(a.d)) {
    case 1: return a.d <= 256 ? launch_gradients<T, VE, 8, 1>(a, parts, s) : launch_gradients<T, VE, 16, 1>(a, parts, s);
    case 2: return launch_gradients<T, VE, 16, 2>(a, parts, s);
    case 4: return launch_gradients<T, VE, 16, 4>(a, parts, s);
    case 8: return launch_gradients<T, VE, 16, 8>(a, parts, s);
    default: return launch_gradients<T, VE, 16, 16>(a, parts, s);
  }
}
template <typename T, int VE, int NV>
cudaError_t launch_few_gradients(const NormArgs& a, cudaStream_t s) {
  const int cols = a.d_weight || a.d_bias ? ceil_div(a.d / VE, kFewCols) : 0;
  return launch(true, norm_backward_few_kernel<T, VE, NV>, cols + (a.d_x ? a.R : 0), kFewThreads, 0, s, a, cols);
}
template <typename T, int VE>
cudaError_t launch_wide_gradients(const NormArgs& a, int parts, cudaStream_t s) {
  cudaError_t e = a.d_x ? launch(true, norm_wide_dx_kernel<T, VE>, a.R, kWideDx, 0, s, a) : cudaSuccess;
  if (e == cudaSuccess && (a.d_weight || a.d_bias))
    e = launch(true, norm_wide_sums_kernel<T, VE>, dim3(ceil_div(a.d / VE, 32), parts), 256, 0, s, a);
  return e;
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
  if (few_gradients(a.R, a.d))
    return by_row_type(a.dtype, a.d, [&](auto t) {
      using Row = decltype(t);
      return a.d <= 2048 ? launch_few_gradients<typename Row::T, Row::VE, 8 / Row::VE>(a, s)
                         : launch_few_gradients<typename Row::T, Row::VE, 32 / Row::VE>(a, s);
    });
  const int parts = part_count(a.R, a.d);
  const cudaError_t e = by_row_type(a.dtype, a.d, [&](auto t) {
    using Row = decltype(t);
    return a.d > kWideCols ? launch_wide_gradients<typename Row::T, Row::VE>(a, parts, s)
                           : launch_gradients<typename Row::T, Row::VE>(a, parts, s);
  });
  if (e != cudaSuccess || (!a.d_weight && !a.d_bias)) return e;
  const dim3 grid(ceil_div(a.d, 32), 2);
  if (parts <= 8 * kJoinAhead) return launch(true, norm_join_kernel<8>, grid, 256, 0, s, a, parts);
  return launch(true, norm_join_kernel<32>, grid, 1024, 0, s, a, parts);
}

}  // namespace cmsd
