// The head's loss and its gradients (include/cmsd.h, cmsd_lmhead_loss and
// cmsd_lmhead_loss_backward).
//
// Forward: the logits of a tile of rows and vocabulary entries are formed in
// registers and reduced at once to each row's maximum and sum of exponentials
// over the tile's entries; a second kernel merges a row's tiles.  Backward, a
// piece of the vocabulary at a time: the logits again, from them the piece of
// P (bf16), then P W, summed over the pieces in fp32, and P^T h.
#include <cuda_bf16.h>

#include "cmsd_device.cuh"
#include "cmsd_head.h"

namespace cmsd {
namespace {

__device__ __forceinline__ float bf(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ uint16_t to_bf(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
__device__ __forceinline__ bool kept(const HeadLossArgs& a, int label) {
  return label != a.ignore && label >= 0 && label < a.V;
}

// ---- the kept rows, packed --------------------------------------------------------
constexpr int kPackThreads = 256;
// Each CTA packs `rows` consecutive rows: it counts the kept rows before its
// own in the labels (a prefix of them, read again by every CTA), then copies.
// The last one also writes the count and fills up to the next whole tile.
__global__ void __launch_bounds__(kPackThreads) head_pack_kernel(const HeadLossArgs a, int rows) {
  __shared__ int s_sum[kPackThreads / 32];
  __shared__ int s_base;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r0 = blockIdx.x * rows, r1 = min(a.R, r0 + rows);
  int c = 0;
  for (int r = tid; r < r0; r += kPackThreads) c += kept(a, a.labels[r]);
  c = __reduce_add_sync(kFull, c);
  if (lane == 0) s_sum[warp] = c;
  __syncthreads();
  if (tid == 0) {
    int b = 0;
    for (int w = 0; w < kPackThreads / 32; ++w) b += s_sum[w];
    s_base = b;
  }
  __syncthreads();
  int base = s_base;
  // one warp a row, in turn
  for (int r = r0; r < r1; r += kPackThreads / 32) {
    // every warp knows the places of the group's rows
    const int mine = r + lane;
    const int label = lane < kPackThreads / 32 && mine < r1 ? a.labels[mine] : a.ignore;
    const bool in = lane < kPackThreads / 32 && mine < r1;
    const unsigned k = __ballot_sync(kFull, in && kept(a, label));
    if (warp == 0 && in) {
      const bool keep = (k >> lane) & 1u;
      const int p = base + __popc(k & ((1u << lane) - 1u));
      a.pos[mine] = keep ? p : -1;
      if (keep) {
        a.lab[p] = label;
        if (a.plse) {
          a.plse[p] = a.lse_in[mine];
          a.pgrad[p] = a.grad[mine];
        }
      } else if (label != a.ignore) {
        atomicOr(a.err, 1u);
      }
    }
    const int row = r + warp;
    if (row < r1 && ((k >> warp) & 1u)) {
      const int p = base + __popc(k & ((1u << warp) - 1u));
      const uint4* src = reinterpret_cast<const uint4*>(a.hidden + (size_t)row * a.d);
      uint4* dst = reinterpret_cast<uint4*>(a.packed + (size_t)p * a.d);
      for (int j = lane; j < a.d / 8; j += 32) dst[j] = src[j];
    }
    base += __popc(k);
  }
  if (r1 == a.R) {
    if (tid == 0) *a.n = base;
    const int end = min(a.Rp, (base + kHeadTile - 1) / kHeadTile * kHeadTile);
    const size_t from = (size_t)base * a.d / 8, to = (size_t)end * a.d / 8;
    for (size_t j = from + tid; j < to; j += kPackThreads) reinterpret_cast<uint4*>(a.packed)[j] = make_uint4(0, 0, 0, 0);
    for (int p = base + tid; p < end; p += kPackThreads) {
      a.lab[p] = -1;
      if (a.plse) {
        a.plse[p] = 0.f;
        a.pgrad[p] = 0.f;
      }
    }
  }
}

// ---- the products ---------------------------------------------------------------------
enum Op { kOpStats, kOpDz, kOpDh, kOpDw };
constexpr int kTM = 64, kTN = 128, kTK = 16;

// v0, vlen: the piece of the vocabulary; first: the first piece
template <int OP>
__global__ void __launch_bounds__(256) head_gemm_kernel(const HeadLossArgs a, int v0, int vlen, int first) {
  __shared__ float sa[kTK][kTM + 4], sb[kTK][kTN + 4];
  __shared__ float s_m[kTM][17], s_s[kTM][17];
  const int n = *a.n;
  const int M = OP == kOpDw ? vlen : n, N = OP == kOpStats || OP == kOpDz ? vlen : a.d;
  const int K = OP == kOpStats || OP == kOpDz ? a.d : (OP == kOpDh ? vlen : n);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int n0 = blockIdx.x * kTN;
  const int Mt = OP == kOpDz ? (M + kHeadTile - 1) / kHeadTile * kHeadTile : M;
  for (int m0 = blockIdx.y * kTM; m0 < Mt; m0 += gridDim.y * kTM) {
    float acc[4][8] = {};
    for (int k0 = 0; k0 < K; k0 += kTK) {
      __syncthreads();
      for (int e = tid; e < kTK * kTM; e += 256) {
        const int k = e % kTK, m = e / kTK;
        float x = 0.f;
        if (m0 + m < M && k0 + k < K) {
          const size_t i = m0 + m, j = k0 + k;
          x = bf(OP == kOpDh ? a.dz[i * a.Vc + j] : (OP == kOpDw ? a.dz[j * a.Vc + i] : a.packed[i * a.d + j]));
        }
        sa[k][m] = x;
      }
      for (int e = tid; e < kTK * kTN; e += 256) {
        const int k = e % kTK, m = e / kTK;
        float x = 0.f;
        if (n0 + m < N && k0 + k < K) {
          const size_t i = n0 + m, j = k0 + k;
          x = bf(OP == kOpDh ? a.weight[(v0 + j) * a.d + i]
                             : (OP == kOpDw ? a.packed[j * a.d + i] : a.weight[(v0 + i) * a.d + j]));
        }
        sb[k][m] = x;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kTK; ++k)
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int t = 0; t < 8; ++t) acc[u][t] = fmaf(sa[k][ty * 4 + u], sb[k][tx + 16 * t], acc[u][t]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int m = m0 + ty * 4 + u;
      if (OP == kOpStats) {
        float mx = -pos_inf(), s = 0.f;
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (n0 + tx + 16 * t < N) mx = fmaxf(mx, acc[u][t] * kLog2e);
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (n0 + tx + 16 * t < N) {
            s += ex2(acc[u][t] * kLog2e - mx);
            if (m < M && a.lab[m] == n0 + tx + 16 * t) a.zlab[m] = acc[u][t];
          }
        s_m[ty * 4 + u][tx] = mx;
        s_s[ty * 4 + u][tx] = s;
      } else if (m < Mt) {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const int j = n0 + tx + 16 * t;
          if (OP == kOpDz) {
            float p = 0.f;
            if (m < M && j < N)
              p = (ex2((acc[u][t] - a.plse[m]) * kLog2e) - (a.lab[m] == v0 + j ? 1.f : 0.f)) * a.pgrad[m];
            if (j < a.Vc) a.dz[(size_t)m * a.Vc + j] = to_bf(p);
          } else if (j < N) {
            if (OP == kOpDh) {
              float* p = a.dh + (size_t)m * a.d + j;
              *p = first ? acc[u][t] : *p + acc[u][t];
            } else {
              a.d_weight[(size_t)(v0 + m) * a.d + j] = to_bf(acc[u][t]);
            }
          }
        }
      }
    }
    if (OP == kOpStats) {
      __syncthreads();
      if (tid < kTM && m0 + tid < M) {
        float mx = -pos_inf(), s = 0.f;
        for (int t = 0; t < 16; ++t) mx = fmaxf(mx, s_m[tid][t]);
        for (int t = 0; t < 16; ++t) s += s_s[tid][t] > 0.f ? s_s[tid][t] * ex2(s_m[tid][t] - mx) : 0.f;
        a.part[(size_t)blockIdx.x * a.Rp + m0 + tid] = make_float2(mx, s);
      }
    }
  }
}

// ---- a row's tiles merged -----------------------------------------------------------
__global__ void __launch_bounds__(256) head_merge_kernel(const HeadLossArgs a, int parts) {
  const int lane = threadIdx.x & 31;
  const int r = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (r >= a.R) return;
  const int p = a.pos[r];
  float lse = 0.f, loss = 0.f;
  if (p >= 0) {
    float m = -pos_inf(), s = 0.f;
    for (int t = lane; t < parts; t += 32) {
      const float2 x = a.part[(size_t)t * a.Rp + p];
      const float mm = fmaxf(m, x.x);
      s = s * ex2(m - mm) + x.y * ex2(x.x - mm);
      m = mm;
    }
    for (int o = 16; o; o >>= 1) {
      const float m2 = __shfl_xor_sync(kFull, m, o), s2 = __shfl_xor_sync(kFull, s, o);
      const float mm = fmaxf(m, m2);
      s = (s > 0.f ? s * ex2(m - mm) : 0.f) + (s2 > 0.f ? s2 * ex2(m2 - mm) : 0.f);
      m = mm;
    }
    lse = m * kLn2 + logf(s);
    loss = lse - a.zlab[p];
  }
  if (lane == 0) {
    a.lse[r] = lse;
    if (a.loss) a.loss[r] = loss;
  }
}

// ---- the hidden states' gradient, rounded and put back in place -------------------
__global__ void __launch_bounds__(256) head_unpack_kernel(const HeadLossArgs a) {
  const int lane = threadIdx.x & 31;
  const int r = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (r >= a.R) return;
  const int p = a.pos[r];
  for (int j = lane; j < a.d; j += 32) {
    float x = 0.f;
    if (p >= 0)
      for (int k = 0; k < a.split; ++k) x += a.dh[((size_t)k * a.Rp + p) * a.d + j];
    a.d_hidden[(size_t)r * a.d + j] = to_bf(x);
  }
}

unsigned tiles(int64_t n, int t) { return (unsigned)((n + t - 1) / t); }
cudaError_t launch_pack(const HeadLossArgs& a, cudaStream_t s) {
  int rows = 16;
  while ((int64_t)rows * 1024 < a.R) rows *= 2;
  head_pack_kernel<<<tiles(a.R, rows), kPackThreads, 0, s>>>(a, rows);
  return cudaGetLastError();
}
}  // namespace

int head_split(int Rp, int d, int Vc) { return 1; }

cudaError_t launch_head_loss(const HeadLossArgs& a, cudaStream_t s) {
  cudaError_t e = launch_pack(a, s);
  if (e != cudaSuccess) return e;
  const unsigned my = min(tiles(a.R, kTM), 65535u);
  head_gemm_kernel<kOpStats><<<dim3(tiles(a.V, kTN), my), 256, 0, s>>>(a, 0, a.V, 1);
  head_merge_kernel<<<tiles(a.R, 8), 256, 0, s>>>(a, (int)tiles(a.V, kTN));
  return cudaGetLastError();
}

cudaError_t launch_head_loss_backward(const HeadLossArgs& a, cudaStream_t s) {
  cudaError_t e = launch_pack(a, s);
  if (e != cudaSuccess) return e;
  const unsigned my = min(tiles(a.Rp, kTM), 65535u);
  for (int64_t v0 = 0; v0 < a.V; v0 += a.Vc) {
    const int vlen = (int)min((int64_t)a.Vc, a.V - v0);
    head_gemm_kernel<kOpDz><<<dim3(tiles(a.Vc, kTN), my), 256, 0, s>>>(a, (int)v0, vlen, 0);
    if (a.d_hidden)
      head_gemm_kernel<kOpDh><<<dim3(tiles(a.d, kTN), my), 256, 0, s>>>(a, (int)v0, vlen, v0 == 0);
    if (a.d_weight)
      head_gemm_kernel<kOpDw><<<dim3(tiles(a.d, kTN), min(tiles(vlen, kTM), 65535u)), 256, 0, s>>>(a, (int)v0, vlen, 0);
  }
  if (a.d_hidden) head_unpack_kernel<<<tiles(a.R, 8), 256, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace cmsd
