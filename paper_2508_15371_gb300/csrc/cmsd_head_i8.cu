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
constexpr int kQuantThreads = 256;

// 127 x / a rounded to the nearest whole number, ties to the even one, exactly:
// the quotient by r ~ 1 / a decides unless it lies within 2^-12 of a tie (it is
// off by less than 127 * 2^-21); there the sign of 127 x - c a, c the tie, does,
// from the two products' roundings (each product's error is one fma, and the
// difference of the rounded products is exact, as they are within a factor of
// two of each other).  0 <= x <= a, both scaled so that nothing overflows.
__device__ __forceinline__ float quantize_abs(float x, float a, float r) {
  const float hi = __fmul_rn(127.f, x);
  const float t = hi * r;
  float q = rintf(t);
  const float f = fabsf(t - q);
  if (f > 0.5f - 0x1p-12f) {
    const float k = floorf(t), c = k + 0.5f;
    const float lo = __fmaf_rn(127.f, x, -hi);
    const float ph = __fmul_rn(c, a), pl = __fmaf_rn(c, a, -ph);
    const float past = (hi - ph) + (lo - pl);
    const bool odd = ((int)k & 1) != 0;
    q = past > 0.f || (past == 0.f && odd) ? k + 1.f : k;
  }
  return q;
}

__device__ __forceinline__ float load_f(const float* p, size_t i) { return p[i]; }
__device__ __forceinline__ float load_f(const __nv_bfloat16* p, size_t i) { return __bfloat162float(p[i]); }

template <typename T>
__global__ void __launch_bounds__(kQuantThreads) quantize_kernel(const T* __restrict__ x, int R, int d,
                                                                 int8_t* __restrict__ q, float* __restrict__ scale) {
  __shared__ uint32_t s_max[kQuantThreads / 32];
  const int tid = threadIdx.x;
  for (int r = blockIdx.x; r < R; r += gridDim.x) {
    const T* row = x + (size_t)r * d;
    // the bits of |x| order like its value, an infinity and then NaNs on top
    uint32_t m = 0;
    for (int j = tid; j < d; j += kQuantThreads) m = max(m, __float_as_uint(load_f(row, j)) & 0x7FFFFFFFu);
    m = __reduce_max_sync(kFull, m);
    if ((tid & 31) == 0) s_max[tid >> 5] = m;
    __syncthreads();
    for (int w = 0; w < kQuantThreads / 32; ++w) m = max(m, s_max[w]);
    __syncthreads();
    const float a0 = __uint_as_float(m);
    const bool fine = m != 0 && m < 0x7F800000u;
    const float f = a0 < 0x1p-60f ? 0x1p100f : (a0 > 0x1p60f ? 0x1p-100f : 1.f);
    const float a = fine ? a0 * f : 1.f, inv = 1.f / a;
    for (int j = tid; j < d; j += kQuantThreads) {
      const float v = load_f(row, j);
      const float u = fine ? quantize_abs(fabsf(v) * f, a, inv) : 0.f;
      q[(size_t)r * d + j] = (int8_t)(int)copysignf(u, v);
    }
    if (tid == 0) scale[r] = __fdiv_rn(a0, 127.f);
  }
}

// ---- the product ----------------------------------------------------------------
//
// A whole number of 8 bits is exact in fp16, its products are exact in the
// tensor cores and their sums exact in fp32 up to 2^24: 1024 products of at
// most 2^14.  So the integers go through the fp16 tensor cores (GB300's integer
// tensor rate is far below), and the sums of each 1024 entries of K are added
// up as 32-bit integers.  Only the 8-bit weight is read from memory; its bytes
// become fp16 on their way into tensor memory, where the MMA takes its A from:
// byte + 128 is placed into the low mantissa bits of 1024.0, and 1152 is
// subtracted, both exact.
//
// The MMA's M is the vocabulary (a tile of up to 256 entries: two accumulators
// of 128 lanes) and its N the tokens (up to 128), so the weight, the large
// operand, passes through registers once, and B's tile serves both accumulators.
//   warp 0      lane 0 fills the ring: 128 bytes of K of the tile's weight rows,
//               and the same K of the tokens (fp16, from the workspace);
//   warp 1      lane 0 issues the MMAs;
//   warps 2..9  thread = one vocabulary entry: turns its row of a stage into
//               fp16, and adds up and scales its row of sums.  The first stage
//               of the next 1024 of K is turned before the sums of the last are
//               read, so that the MMAs resume at once.
// Barriers: full (TMA -> fp16 and MMA), afull / aempty (fp16 <-> MMA, two
// buffers in tensor memory), empty (MMA -> TMA), dfull / dempty (MMA <-> sums).
// Every wait is bounded.
constexpr int kI8Tile = 256;                        // vocabulary entries per tile at most
constexpr int kI8K = 128;                           // K per stage
constexpr int kI8Exact = 1024 / kI8K;               // stages whose sums are exact in fp32
constexpr int kI8Threads = 64 + kI8Tile;
constexpr int kI8WStage = kI8Tile * kI8K;
template <int NT>
struct I8Shape {
  static constexpr int kHStage = NT * kI8K * 2;
  static constexpr int kStage = kI8WStage + kHStage;
  static constexpr int kStages = NT == 128 ? 3 : (NT == 64 ? 4 : 5);
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kStage + 8 * (2 * kStages + 6) + 16;
  static_assert(kSmem <= 227 * 1024, "shared memory");
};
__device__ __forceinline__ float ld_volatile_f(const float* p) {
  float x;
  asm volatile("ld.global.f32 %0, [%1];" : "=f"(x) : "l"(p) : "memory");
  return x;
}
struct I8Plan {
  int height;            // vocabulary entries per tile (a multiple of 8)
  int cols;              // tokens per tile (a multiple of 16, at most 128)
  int vt, rt;            // tiles of the vocabulary and of the tokens
};

__global__ void __launch_bounds__(256) head_i8_tokens_kernel(const HeadI8Args a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const size_t n = (size_t)a.R * a.d / 16;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    const uint4 x = reinterpret_cast<const uint4*>(a.hidden)[i];
    uint32_t h[8];
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) i8_to_half(w[k], h[2 * k], h[2 * k + 1]);
    uint4* dst = reinterpret_cast<uint4*>(a.h16) + 2 * i;
    dst[0] = make_uint4(h[0], h[1], h[2], h[3]);
    dst[1] = make_uint4(h[4], h[5], h[6], h[7]);
  }
}

template <int NT, bool kBf16>
__global__ void __launch_bounds__(kI8Threads, 1)
    head_i8_kernel(const HeadI8Args a, const I8Plan p, const __grid_constant__ CUtensorMap map_w,
                   const __grid_constant__ CUtensorMap map_h) {
  using S = I8Shape<NT>;
  constexpr int kStages = S::kStages;
  extern __shared__ __align__(1024) unsigned char i8_smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t raw = smem_addr(i8_smem);
  const uint32_t base = (raw + 1023u) & ~1023u;
  const uint32_t bars = base + kStages * S::kStage;
  const uint32_t full = bars, empty = bars + 8 * kStages, afull = bars + 16 * kStages, aempty = afull + 16;
  const uint32_t dfull = afull + 32, dempty = afull + 40;
  uint32_t* s_taddr = reinterpret_cast<uint32_t*>(i8_smem + (bars - raw) + 8 * (2 * kStages + 6));
  if (tid == 0) {
    for (int k = 0; k < kStages; ++k) {
      mbar_init(full + 8 * k, 1);
      mbar_init(empty + 8 * k, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(afull + 8 * b, 8);
      mbar_init(aempty + 8 * b, 1);
    }
    mbar_init(dfull, 1);
    mbar_init(dempty, 8);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(s_taddr)),
                 "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tbase = *s_taddr;
  const uint32_t abase = tbase + 256;               // two buffers of two blocks of 64 columns
  const int ks = (a.d + kI8K - 1) / kI8K;           // stages per tile
  const int tiles = p.vt * p.rt;
  const int mine = tiles > (int)blockIdx.x ? (tiles - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x : 0;
  const int G = mine * ks;
  bool ok = true;

  if (warp == 0) {
    if (lane == 0) {
      const uint32_t bytes = (uint32_t)(p.height * kI8K + p.cols * kI8K * 2);
      // the weight's first stages do not wait for the tokens' kernel: it has
      // started, so what precedes it on the stream has ended
      int issued = G < kStages ? G : kStages;
      for (int g = 0; g < issued; ++g) {
        const int t = (int)blockIdx.x + g / ks * (int)gridDim.x;
        mbar_arrive_tx(full + 8 * g, bytes);
        tma_box(base + g * S::kStage, &map_w, g % ks * kI8K, t / p.rt * p.height, full + 8 * g);
      }
      asm volatile("griddepcontrol.wait;" ::: "memory");
      asm volatile("fence.proxy.async.global;" ::: "memory");
      for (int g = 0; g < G; ++g) {
        const int s = g % kStages, t = (int)blockIdx.x + g / ks * (int)gridDim.x, k = g % ks * kI8K;
        const int v = t / p.rt, r = t - v * p.rt;
        const uint32_t dst = base + s * S::kStage;
        if (g >= kStages) {
          if (ok) ok = mbar_wait(empty + 8 * s, (uint32_t)((g / kStages - 1) & 1));
          mbar_arrive_tx(full + 8 * s, bytes);
          tma_box(dst, &map_w, k, v * p.height, full + 8 * s);
        }
        tma_box(dst + kI8WStage, &map_h, k, r * p.cols, full + 8 * s);
        tma_box(dst + kI8WStage + p.cols * 128, &map_h, k + 64, r * p.cols, full + 8 * s);
      }
      // nothing is in flight into this CTA when it ends
      for (int g = (G > kStages ? G - kStages : 0); g < G; ++g)
        if (ok) ok = mbar_wait(empty + 8 * (g % kStages), (uint32_t)((g / kStages) & 1));
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = mma_idesc(128, p.cols, false, false, false);
      int c = 0;                                    // sums handed over
      for (int g = 0; g < G; ++g) {
        const int s = g % kStages, b = g & 1, k = g % ks;
        if (k % kI8Exact == 0) {
          if (c > 0 && ok) ok = mbar_wait(dempty, (uint32_t)((c - 1) & 1));
        }
        if (ok) ok = mbar_wait(full + 8 * s, (uint32_t)((g / kStages) & 1));
        if (ok) ok = mbar_wait(afull + 8 * b, (uint32_t)((g / 2) & 1));
        tmem_fence_after();
        const uint32_t hs = base + s * S::kStage + kI8WStage;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          if (sub * 128 >= p.height) break;
#pragma unroll
          for (int j = 0; j < kI8K / 16; ++j)
            mma_tmem_a(tbase + sub * 128, abase + b * 128 + sub * 64 + j * 8,
                       mma_desc(hs + (j >> 2) * p.cols * 128, 0) + (uint64_t)(2 * (j & 3)), idesc,
                       (k % kI8Exact) != 0 || j != 0);
        }
        mma_commit(aempty + 8 * b);
        mma_commit(empty + 8 * s);
        if (k % kI8Exact == kI8Exact - 1 || k == ks - 1) {
          mma_commit(dfull);
          ++c;
        }
      }
    }
    __syncwarp();
  } else {
    const int q = warp & 3, sub = (warp - 2) >> 2;
    const int row = sub * 128 + q * 32 + lane;      // vocabulary entry within the tile
    const uint32_t quarter = (uint32_t)(q * 32) << 16;
    const uint32_t wrow = (uint32_t)row * 128, x8 = (uint32_t)(row & 7);
    int acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = 0;
    int c = 0, due = -1;                            // stage whose sums are to be read next, -1: none
    bool waited = false;
    for (int g = 0; g <= G; ++g) {
      if (g < G) {
        const int s = g % kStages, b = g & 1;
        if (ok) ok = mbar_wait(full + 8 * s, (uint32_t)((g / kStages) & 1));
        if (g >= 2 && ok) ok = mbar_wait(aempty + 8 * b, (uint32_t)((g / 2 - 1) & 1));
        __syncwarp();
        tmem_fence_after();
        const uint32_t src = base + s * S::kStage + wrow;
        // 64 columns, as many at a time as registers are left beside the sums
        constexpr int kCols = NT == 128 ? 16 : 32;
#pragma unroll
        for (int h = 0; h < 64 / kCols; ++h) {
          uint32_t o[kCols];
#pragma unroll
          for (int j = 0; j < kCols / 8; ++j) {
            uint32_t w0, w1, w2, w3;
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(w0), "=r"(w1), "=r"(w2), "=r"(w3)
                         : "r"(src + ((((uint32_t)(h * (kCols / 8) + j)) ^ x8) << 4)));
            i8_to_half(w0, o[8 * j], o[8 * j + 1]);
            i8_to_half(w1, o[8 * j + 2], o[8 * j + 3]);
            i8_to_half(w2, o[8 * j + 4], o[8 * j + 5]);
            i8_to_half(w3, o[8 * j + 6], o[8 * j + 7]);
          }
          tmem_st(abase + quarter + b * 128 + sub * 64 + kCols * h, o);
        }
        tmem_st_wait();
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_local(afull + 8 * b);
      }
      // the sums that ended at the stage before this one
      if (due >= 0) {
        if (ok) ok = mbar_wait(dfull, (uint32_t)(c & 1));
        ++c;
        __syncwarp();
        tmem_fence_after();
#pragma unroll
        for (int n = 0; n < NT; n += 16) {
          if (n < p.cols) {
            float z[16];
            tmem_ld16(tbase + quarter + sub * 128 + n, z);
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[n + j] += __float2int_rn(z[j]);
          }
        }
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_local(dempty);
        if (due % ks == ks - 1) {                   // the tile's last: scaled and written
          if (!waited) {                            // what the call before may still read or write
            asm volatile("griddepcontrol.wait;" ::: "memory");
            waited = true;
          }
          const int t = (int)blockIdx.x + due / ks * (int)gridDim.x;
          const int vi = t / p.rt, r0 = (t - vi * p.rt) * p.cols;
          const int v = vi * p.height + row;
          if (row < p.height && v < a.V) {
            const float ws = a.weight_scale[v];
#pragma unroll
            for (int n0 = 0; n0 < NT; n0 += 16) {
              if (n0 < p.cols) {
                float hs[16];                       // (sixteen at a time: more would cost the sums their registers)
#pragma unroll
                for (int j = 0; j < 16; ++j) hs[j] = ld_volatile_f(a.hidden_scale + min(r0 + n0 + j, a.R - 1));
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                  const int r = r0 + n0 + j;
                  const float z = (float)acc[n0 + j] * hs[j] * ws;
                  if (r < a.R) {
                    const size_t at = (size_t)r * a.V + v;
                    if (kBf16)
                      reinterpret_cast<__nv_bfloat16*>(a.logits)[at] = __float2bfloat16_rn(z);
                    else
                      reinterpret_cast<float*>(a.logits)[at] = z;
                  }
                }
              }
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) acc[n] = 0;
        }
      }
      due = g < G && ((g % ks) % kI8Exact == kI8Exact - 1 || g % ks == ks - 1) ? g : -1;
    }
  }
  if (!ok) atomicOr(a.err, 4u);
  __syncwarp();
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tbase), "r"(512) : "memory");
}

template <int NT, bool kBf16>
cudaError_t launch_i8(const HeadI8Args& a, const I8Plan& p, int grid, int dev, const CUtensorMap& mw,
                      const CUtensorMap& mh, cudaStream_t s) {
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
  return cudaLaunchKernelEx(&cfg, head_i8_kernel<NT, kBf16>, a, p, mw, mh);
}
template <bool kBf16>
cudaError_t launch_i8_cols(const HeadI8Args& a, const I8Plan& p, int grid, int dev, const CUtensorMap& mw,
                           const CUtensorMap& mh, cudaStream_t s) {
  if (p.cols <= 16) return launch_i8<16, kBf16>(a, p, grid, dev, mw, mh, s);
  if (p.cols <= 32) return launch_i8<32, kBf16>(a, p, grid, dev, mw, mh, s);
  if (p.cols <= 64) return launch_i8<64, kBf16>(a, p, grid, dev, mw, mh, s);
  return launch_i8<128, kBf16>(a, p, grid, dev, mw, mh, s);
}
}  // namespace

cudaError_t launch_quantize_rows(const void* x, int dtype, int R, int d, int8_t* q, float* scale, cudaStream_t s) {
  const int grid = R < (1 << 20) ? R : 1 << 20;
  if (dtype == 0)
    quantize_kernel<float><<<grid, kQuantThreads, 0, s>>>((const float*)x, R, d, q, scale);
  else
    quantize_kernel<__nv_bfloat16><<<grid, kQuantThreads, 0, s>>>((const __nv_bfloat16*)x, R, d, q, scale);
  return cudaGetLastError();
}

cudaError_t launch_head_i8(const HeadI8Args& a, cudaStream_t s) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  if (sms < 1) sms = 1;
  I8Plan p;
  p.rt = (a.R + 127) / 128;
  p.cols = ((a.R + p.rt - 1) / p.rt + 15) / 16 * 16;
  p.rt = (a.R + p.cols - 1) / p.cols;
  // one tile of tokens: the weight is streamed once, so its rows are spread
  // evenly over the SMs; more of them: whole tiles
  const int64_t wave = (int64_t)sms * kI8Tile;
  const int64_t waves = (a.V + wave - 1) / wave;
  p.height = p.rt > 1 ? kI8Tile : (int)(((a.V + sms * waves - 1) / (sms * waves) + 7) / 8 * 8);
  p.vt = (a.V + p.height - 1) / p.height;
  CUtensorMap mw, mh;
  if (!tma_matrix(&mw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.weight, a.d, a.V, p.height) ||
      !tma_matrix(&mh, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, a.h16, a.d, a.R, p.cols))
    return cudaErrorInvalidValue;
  const int64_t n16 = (int64_t)a.R * a.d / 16;
  head_i8_tokens_kernel<<<(unsigned)(n16 < 256 * 2048 ? (n16 + 255) / 256 : 2048), 256, 0, s>>>(a);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const int64_t tiles = (int64_t)p.vt * p.rt;
  const int grid = tiles < sms ? (int)tiles : sms;
  return a.dtype == 0 ? launch_i8_cols<false>(a, p, grid, dev, mw, mh, s) : launch_i8_cols<true>(a, p, grid, dev, mw, mh, s);
}

}  // namespace cmsd
