// Scaled rows of the token table (include/cmsd.h, cmsd_embedding) and the
// table's gradient (cmsd_embedding_backward).
//
// Of more than 512 rows the gradient's are put into the order of their tokens first
// (stable: rows of one token keep theirs), by tokens alone, while a table that is not
// added to gets its zeros; then the rows of d_x with a token are read once each, and
// the sums written, over zeros where there are some.  Fewer rows are not put in order:
// one launch reads them, writes the sums, and zeros elsewhere.
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "cmsd_device.cuh"
#include "cmsd_errors.cuh"
#include "cmsd_launch.cuh"
#include "cmsd_rows.cuh"
#include "cmsd_train.h"

namespace cmsd {
namespace {

// ---- rows of the table ------------------------------------------------------------
// A warp a piece of 256 vectors of a row, eight requested at once.  Bound by memory:
// 16384 rows, 11469 with a token, d = 2048 of 128256 bf16 15.6 us, 5.7 TB/s.
constexpr int kAhead = 8;
template <typename T, int VE>
__global__ void __launch_bounds__(256) embed_kernel(const EmbedArgs a, int pieces) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
  wait_for_previous();
  const int lane = threadIdx.x & 31, nvec = a.d / VE;
  const int64_t units = (int64_t)a.R * pieces, step = (int64_t)gridDim.x * (blockDim.x >> 5);
  for (int64_t u = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); u < units; u += step) {
    const int r = (int)(u / pieces), v0 = (int)(u % pieces) * 32 * kAhead + lane;
    const int token = a.tokens[r];
    const bool in = token >= 0 && token < a.V, keep = in && token != a.ignore;
    if (!in && token != a.ignore && v0 == 0) report(nullptr, 1u);
    const Raw* row = static_cast<const Raw*>(a.table) + (size_t)(keep ? token : 0) * nvec;
    Raw* x = static_cast<Raw*>(a.x) + (size_t)r * nvec;
    Raw w[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      w[k] = V::zero();
      if (keep && v0 + 32 * k < nvec) w[k] = row[v0 + 32 * k];
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (v0 + 32 * k < nvec) {
        float f[VE];
        V::get(w[k], f);
#pragma unroll
        for (int j = 0; j < VE; ++j) f[j] *= a.scale;
        x[v0 + 32 * k] = keep ? V::put(f) : V::zero();
      }
  }
}

// Narrow rows, many of them: a warp 256 vectors of x in a row, whatever rows they are of.  R = 32768 d = 64 bf16
// 2.8 us, a warp a row 7.6; R = 600000 18 and 143; R = 16384 d = 512 4.8 and 5.0; 6000 d = 64 2.7 and 2.2.
constexpr int kNarrowVecs = 64, kNarrowRows = 8192;
template <typename T, int VE>
__global__ void __launch_bounds__(256) embed_narrow_kernel(const EmbedArgs a) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
  wait_for_previous();
  const int lane = threadIdx.x & 31, nvec = a.d / VE;
  const int64_t all = (int64_t)a.R * nvec, step = (int64_t)gridDim.x * 256 * kAhead;
  for (int64_t q0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * 32 * kAhead; q0 < all; q0 += step) {
    const int r0 = (int)(q0 / nvec), v0 = (int)(q0 % nvec) + lane;
    int token[kAhead], v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = v0 + 32 * k, r = (int)((unsigned)i / (unsigned)nvec);
      v[k] = q0 + lane + 32 * k < all ? i - r * nvec : -1;
      token[k] = v[k] >= 0 ? a.tokens[r0 + r] : a.ignore;
    }
    Raw w[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const bool in = token[k] >= 0 && token[k] < a.V;
      if (!in && token[k] != a.ignore && v[k] == 0) report(nullptr, 1u);
      if (!in || token[k] == a.ignore) token[k] = -1;
      w[k] = V::zero();
      if (token[k] >= 0) w[k] = static_cast<const Raw*>(a.table)[(size_t)token[k] * nvec + v[k]];
    }
    Raw* x = static_cast<Raw*>(a.x) + q0 + lane;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      float f[VE];
      V::get(w[k], f);
#pragma unroll
      for (int j = 0; j < VE; ++j) f[j] *= a.scale;
      if (v[k] >= 0) x[32 * k] = token[k] >= 0 ? V::put(f) : V::zero();
    }
  }
}

// ---- few rows ----------------------------------------------------------------------------
// All in one launch, nothing put in order: every CTA has all tokens in shared
// memory.  CTAs of kFewTile rows look up which of theirs come first of their token,
// list the rows of those tokens in order, and add them up, the columns over the
// threads; the others write zeros to the rows of kFewFill bytes of the table that
// no token is of.  Bound by memory (R = 333 d = 1000 of 32001 f32 21.1 us, 6.1 TB/s),
// or by the row of loads: tokens, rows, and a batch of them after another where a
// token has many.  Against the three launches below, d = 2048 of 128256 bf16: R = 1
// 69.1 against 71.5 us, 512 70.5 and 75.5; added to a table, d = 1024, R = 256 4.7
// and 6.3, 512 7.2 and 7.7, 1024 11.9 and 8.7: all with frequencies that fall as one
// over the rank.  The rule does not look at the tokens, and one CTA has all rows of
// its tokens: at R = 512 d = 1024 of 32000 with a tenth, half, all rows of one token
// 14.4, 35, 60 us (added 8.7, 23, 41), where 513 rows take 14.6, 15.2, 15.7 (6.5, 6.9, 7.4).
constexpr int kFewRows = 512, kFewTile = 4, kFewThreads = 128, kFewTokens = 1024;
constexpr size_t kFewFill = (size_t)48 << 10;
template <typename T, int VE, bool ADD>
__global__ void __launch_bounds__(kFewThreads) embed_few_kernel(const EmbedArgs a, int tiles, int chunks, int per) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
  constexpr int kBatch = ADD ? 8 : 16;
  wait_for_previous();
  const int nvec = a.d / VE, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if ((int)blockIdx.x >= tiles * chunks) {
    __shared__ uint8_t s_there[kFewTokens];
    const int64_t v0 = (int64_t)((int)blockIdx.x - tiles * chunks) * per;
    const int n = (int)(a.V - v0 < per ? a.V - v0 : per);
    for (int c = threadIdx.x; c < n; c += kFewThreads) s_there[c] = 0;
    __syncthreads();
    for (int k = threadIdx.x; k < a.R; k += kFewThreads) {
      const int token = a.tokens[k];
      if (token != a.ignore && token >= v0 && token - v0 < n) s_there[token - v0] = 1;
    }
    __syncthreads();
    if constexpr (VE * sizeof(T) == 16) {
      Raw* out = static_cast<Raw*>(a.d_table) + (size_t)v0 * nvec;
      if (nvec >= kFewThreads) {
        for (int c = 0; c < n; ++c)
          if (!s_there[c])
            for (int j = threadIdx.x; j < nvec; j += kFewThreads) out[(size_t)c * nvec + j] = V::zero();
      } else {
        for (int j = threadIdx.x; j < n * nvec; j += kFewThreads)
          if (!s_there[j / nvec]) out[j] = V::zero();
      }
    } else {
      // 16-byte pieces wherever one is of these rows and of none with a sum, entries in the others
      constexpr int kPiece = 16 / (int)sizeof(T);
      const size_t first = (size_t)v0 * a.d;
      if (a.d >= kPiece * kFewThreads / 2) {         // row by row: the pieces within it, and its ends
        for (int c = 0; c < n; ++c) {
          if (s_there[c]) continue;
          const size_t at = first + (size_t)c * a.d;
          T* out = static_cast<T*>(a.d_table) + at;
          const int front = (int)(-at % kPiece), pieces = (a.d - front) / kPiece, back = front + pieces * kPiece;
          for (int j = threadIdx.x; j < pieces; j += kFewThreads)
            *reinterpret_cast<uint4*>(out + front + j * kPiece) = make_uint4(0, 0, 0, 0);
          if ((int)threadIdx.x < front) out[threadIdx.x] = from_float<T>(0.f);
          else if ((int)threadIdx.x >= kFewThreads - kPiece && back + (int)threadIdx.x - (kFewThreads - kPiece) < a.d)
            out[back + threadIdx.x - (kFewThreads - kPiece)] = from_float<T>(0.f);
        }
        return;
      }
      const int lead = (int)(first % kPiece), all = n * a.d;           // (below 2^17: kFewFill bytes, or one row)
      T* out = static_cast<T*>(a.d_table) + first;
      for (int e0 = threadIdx.x * kPiece - lead; e0 < all; e0 += kFewThreads * kPiece) {
        const int begin = e0 > 0 ? e0 : 0, end = e0 + kPiece < all ? e0 + kPiece : all, last = (end - 1) / a.d;
        int c = begin / a.d;
        bool none = true;
        for (int q = c; q <= last; ++q) none = none && !s_there[q];
        if (none && end - begin == kPiece) {
          *reinterpret_cast<uint4*>(out + e0) = make_uint4(0, 0, 0, 0);
        } else {
          for (int e = begin; e < end; ++e) {
            if (e >= (c + 1) * a.d) ++c;
            if (!s_there[c]) out[e] = from_float<T>(0.f);
          }
        }
      }
    }
    return;
  }
  __shared__ int s_token[kFewRows];                   // -1: padding
  __shared__ int2 s_list[kFewRows + 16];              // (row or -1, token to write or -1)
  __shared__ int s_count[kFewTile];
  const int tile = blockIdx.x % tiles, chunk = blockIdx.x / tiles, r0 = tile * kFewTile;
  for (int k = threadIdx.x; k < a.R; k += kFewThreads) {
    const int token = a.tokens[k];
    const bool in = token >= 0 && token < a.V;
    if (!in && token != a.ignore && blockIdx.x == 0) report(a.err, 1u);
    s_token[k] = in && token != a.ignore ? token : -1;
  }
  __syncthreads();
  for (int u = warp; u < kFewTile; u += kFewThreads / 32) {
    const int r = r0 + u, token = r < a.R ? s_token[r] : -1;
    int n = 0;
    if (token >= 0) {
      bool first = true;
      for (int k = lane; k - lane < a.R; k += 32) {
        const unsigned same = __ballot_sync(kFull, k < a.R && s_token[k] == token);
        const int before = r - (k - lane);            // lanes of rows before r
        first = first && !(same & (before >= 32 ? kFull : before > 0 ? (1u << before) - 1u : 0u));
        n += __popc(same);
      }
      if (!first) n = 0;
    }
    if (lane == 0) s_count[u] = n;
  }
  __syncthreads();
  int total = 0;
  for (int u = 0; u < kFewTile; ++u) {
    const int n = s_count[u];
    if (u % (kFewThreads / 32) == warp && n > 0) {
      const int token = s_token[r0 + u];
      int at = total;
      for (int k = (r0 + u) / 32 * 32 + lane; k - lane < a.R; k += 32) {
        const bool mine = k < a.R && s_token[k] == token;
        const unsigned same = __ballot_sync(kFull, mine);
        const int p = at + __popc(same & ((1u << lane) - 1u));
        if (mine) s_list[p] = make_int2(k, p == total + n - 1 ? token : -1);
        at += __popc(same);
      }
    }
    total += n;
  }
  if (total == 0) return;                             // (the same in every thread)
  if (threadIdx.x < 16) s_list[total + threadIdx.x] = make_int2(-1, -1);
  __syncthreads();
  const int c = chunk * kFewThreads + threadIdx.x;
  if (c >= nvec) return;
  const Raw* d_x = static_cast<const Raw*>(a.d_x) + c;
  Raw* out = static_cast<Raw*>(a.d_table) + c;
  float sum[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) sum[j] = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < total; k0 += kBatch) {
    Raw x[kBatch], had[ADD ? kBatch : 1];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int2 o = s_list[k0 + u];
      x[u] = V::zero();
      if (o.x >= 0) x[u] = d_x[(size_t)o.x * nvec];
      if (ADD && o.y >= 0) had[u] = out[(size_t)o.y * nvec];
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int token = s_list[k0 + u].y;
      float f[VE];
      V::get(x[u], f);
#pragma unroll
      for (int j = 0; j < VE; ++j) sum[j] += f[j];
      if (token >= 0) {
        if (ADD) V::get(had[ADD ? u : 0], f);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          f[j] = ADD ? __fmaf_rn(sum[j], a.scale, f[j]) : sum[j] * a.scale;
          sum[j] = 0.f;
        }
        out[(size_t)token * nvec] = V::put(f);
      }
    }
  }
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
template <typename T, int VE, bool ADD>
cudaError_t launch_few(const EmbedArgs& a, cudaStream_t s) {
  const size_t row = (size_t)a.d * sizeof(T);
  const int tiles = ceil_div(a.R, kFewTile), chunks = ceil_div(a.d / VE, kFewThreads);
  const int per = (int)std::min<size_t>(kFewTokens, std::max<size_t>(1, kFewFill / row));
  return launch(true, embed_few_kernel<T, VE, ADD>, tiles * chunks + (ADD ? 0 : ceil_div(a.V, per)), kFewThreads, 0, s, a, tiles,
                chunks, per);
}

// ---- the rows in their tokens' order ------------------------------------------------
// What a row is ordered by: its token, or V (behind all tokens) for padding.
__device__ __forceinline__ unsigned key_of(const EmbedArgs& a, int token, bool& bad) {
  const bool in = token >= 0 && token < a.V;
  bad = !in && token != a.ignore;
  return in && token != a.ignore ? (unsigned)token : (unsigned)a.V;
}

// A table that is written whole gets its zeros from the launches that put the rows
// in order: that takes a few CTAs some microseconds a launch, and the others write
// all of the table, equal shares of it.  Rows that get a sum are written again, a
// tenth more bytes where 32768 tokens meet a vocabulary of 128256 (d = 2048 bf16:
// 108 us; with the zeros written beside the sums, where a search finds no rows, 136).
// Chunks of 8 KB: of 16, 32 and 64 KB the ordering CTAs wait longer for their loads
// (110, 112, 116 us), of 4 KB launching CTAs is what bounds (170 us).
constexpr int kFillThreads = 256;
constexpr int kFillVecs = 2;                         // 16-byte vectors of a thread
constexpr size_t kFillChunk = (size_t)kFillThreads * kFillVecs * 16;
constexpr size_t kFillCtas = 1 << 24;                // at most
constexpr size_t kManyZeros = (size_t)64 << 20;      // beside which rows are ordered by an early launch, and so many a row
constexpr size_t kManyZerosRow = (size_t)16 << 10;
// bytes [first, last) of the table, by this and `ctas` - 1 other CTAs
__device__ __forceinline__ void fill(const EmbedArgs& a, size_t first, size_t last, int cta, int ctas) {
  char* table = static_cast<char*>(a.d_table);
  for (size_t chunk = first + (size_t)cta * kFillChunk; chunk < last; chunk += (size_t)ctas * kFillChunk) {
    const size_t at = chunk + threadIdx.x * 16;
#pragma unroll
    for (int k = 0; k < kFillVecs; ++k) {
      const size_t o = at + (size_t)k * kFillThreads * 16;
      if (o + 16 <= last) *reinterpret_cast<uint4*>(table + o) = make_uint4(0, 0, 0, 0);
      else                                           // (the end of a table of odd rows)
        for (size_t q = o; q < last; q += 2) *reinterpret_cast<uint16_t*>(table + q) = 0;
    }
  }
}

// Few rows: each row's place is the number of rows before it in (token, row)
// order, counted by comparing it with all of them: R^2 comparisons of two
// instructions, spread over the GPU, in one launch.  A warp RPW rows, a lane every
// 32nd four of the others.  The whole gradient, R x 1024 of 32000 bf16 added to:
// R = 4096 11.9 us (in passes of the radix sort below 16.9), 6000 15.1 (17.3), 8192
// 18.6 (18.4); written whole 18.8 (20.7), 21.0 (22.1), 24.4 (22.9).
constexpr int kRankRows = 7168;
constexpr int kRankThreads = 256;
constexpr int kRankAhead = 16;                       // tokens of a thread requested at once
template <int RPW>
__global__ void __launch_bounds__(kRankThreads) embed_rank_kernel(const EmbedArgs a, int row_ctas) {
  extern __shared__ uint4 s_key4[];
  unsigned* s_key = reinterpret_cast<unsigned*>(s_key4);
  wait_for_previous();
  if ((int)blockIdx.x >= row_ctas) {
    fill(a, a.fill[0], a.fill[1], blockIdx.x - row_ctas, gridDim.x - row_ctas);
    return;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, padded = (a.R + 127) / 128 * 128;
  for (int rb = threadIdx.x; rb < padded; rb += kRankThreads * kRankAhead) {
    int token[kRankAhead];
#pragma unroll
    for (int u = 0; u < kRankAhead; ++u) {
      const int r = rb + u * kRankThreads;
      token[u] = r < a.R ? a.tokens[r] : 0;
    }
#pragma unroll
    for (int u = 0; u < kRankAhead; ++u) {
      const int r = rb + u * kRankThreads;
      if (r >= padded) break;
      bool bad;
      const unsigned k = key_of(a, token[u], bad);
      if (r < a.R && bad && blockIdx.x == 0) report(a.err, 1u);
      s_key[r] = r < a.R ? k : 0x7FFFFFFFu;
    }
  }
  __syncthreads();
  const int r0 = (blockIdx.x * (kRankThreads / 32) + warp) * RPW;
  if (r0 >= a.R) return;
  unsigned key[RPW];
  int n[RPW];
#pragma unroll
  for (int j = 0; j < RPW; ++j) {
    key[j] = s_key[min(r0 + j, a.R - 1)];
    n[j] = 0;
  }
  // rows before: not above; rows behind: below.  Keys are below 2^31, so a difference's sign bit tells
  const auto below = [](const uint4& t, unsigned k) {
    return (int)((t.x - k >> 31) + (t.y - k >> 31) + (t.z - k >> 31) + (t.w - k >> 31));
  };
  const int own = r0 / 128, all = padded / 128;
#pragma unroll 4
  for (int c = 0; c < own; ++c) {
    const uint4 t = s_key4[c * 32 + lane];
#pragma unroll
    for (int j = 0; j < RPW; ++j) n[j] += below(t, key[j] + 1);
  }
#pragma unroll 4
  for (int c = own + 1; c < all; ++c) {
    const uint4 t = s_key4[c * 32 + lane];
#pragma unroll
    for (int j = 0; j < RPW; ++j) n[j] += below(t, key[j]);
  }
  const uint4 t = s_key4[own * 32 + lane];
  const int at = own * 128 + lane * 4;
#pragma unroll
  for (int j = 0; j < RPW; ++j) {
    const unsigned k = key[j];
    const int r = r0 + j;
    n[j] += (t.x < k + (at < r)) + (t.y < k + (at + 1 < r)) + (t.z < k + (at + 2 < r)) + (t.w < k + (at + 3 < r));
    const int place = __reduce_add_sync(kFull, n[j]);
    if (lane == 0 && r < a.R) {
      a.key[0][place] = k;
      a.order[0][place] = r;
    }
  }
}

// Many rows: a stable radix sort, kRadixBits at most of the key a pass.  Each CTA
// has `tile` consecutive rows, each of its warps an eighth of them.  The first
// pass's counts for each (tile, digit) are made by a kernel of their own, the next
// ones' while the rows are moved (the digit of the next pass, counted for the tile
// that a row moves to: whole numbers, so atomics in any order give the same).
// The three launches of 32768 rows and 128256 tokens take 27 us by themselves, 80 with
// 525 MB of zeros, which take 77 at a copy's rate.
constexpr int kRadixBits = 10;
constexpr int kRadixThreads = 256, kRadixWarps = kRadixThreads / 32;
// Tiles of fewer rows where there are few, so that more SMs take part while a batch or two still has all tiles' counts.
// R x d of V: 8192 x 1024 of 32000 with tiles of 512 22.5 us, of 1024 23.4; 16384 26.8 and 27.8; 25000 x 1024 of 5000 with
// 1024 30.0, with 2048 31.9; 32768 of 1000 29.7 and 28.8.
constexpr int kTileMin = 2048, kShortRows = 16384;
constexpr int kRound = 8;                            // rows of a lane requested at once
constexpr int kCountsAhead = 32;                     // counts of a thread (one by one, 20000 rows of 64 took 30.5 us, not 22.6)
__global__ void __launch_bounds__(kRadixThreads) embed_count_kernel(const EmbedArgs a, int digits, int tiles) {
  extern __shared__ int s_count[];
  wait_for_previous();
  if ((int)blockIdx.x >= tiles) {
    fill(a, a.fill[0], a.fill[1], blockIdx.x - tiles, gridDim.x - tiles);
    return;
  }
  for (int g = threadIdx.x; g < digits; g += kRadixThreads) s_count[g] = 0;
  __syncthreads();
  const int64_t r0 = (int64_t)blockIdx.x * a.tile, r1 = r0 + a.tile < a.R ? r0 + a.tile : a.R;
  for (int64_t rb = r0 + threadIdx.x; rb < r1; rb += kRadixThreads * kRound) {
    int token[kRound];
#pragma unroll
    for (int u = 0; u < kRound; ++u) token[u] = rb + u * kRadixThreads < r1 ? a.tokens[rb + u * kRadixThreads] : 0;
#pragma unroll
    for (int u = 0; u < kRound; ++u) {
      if (rb + u * kRadixThreads >= r1) break;
      bool bad;
      const unsigned k = key_of(a, token[u], bad);
      if (bad) report(a.err, 1u);
      atomicAdd(&s_count[k & (digits - 1)], 1);
    }
  }
  __syncthreads();
  for (int g = threadIdx.x; g < digits; g += kRadixThreads) {
    a.count[0][(size_t)blockIdx.x * digits + g] = s_count[g];
    for (int p = 1; p < a.passes; ++p) a.count[p][(size_t)blockIdx.x * digits + g] = 0;
  }
}

// the CTA's exclusive sum of v over its threads
__device__ __forceinline__ int cta_scan(int v) {
  __shared__ int s_warp[kRadixWarps];
  const int lane = threadIdx.x & 31;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(kFull, s, o);
    if (lane >= o) s += t;
  }
  if (lane == 31) s_warp[threadIdx.x >> 5] = s;
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int w = 0; w < kRadixWarps; ++w) base += w < (int)(threadIdx.x >> 5) ? s_warp[w] : 0;
  return base + s - v;
}

template <bool FIRST>
__global__ void __launch_bounds__(kRadixThreads) embed_move_kernel(const EmbedArgs a, int pass, int bits, int tiles) {
  extern __shared__ int s_at[];                       // [kRadixWarps][digits]: counts, then the next place of each
  const int digits = 1 << bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if ((int)blockIdx.x >= tiles) {                     // (nothing that the launch before makes is used)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    fill(a, a.fill[pass + 1], a.fill[pass + 2], blockIdx.x - tiles, gridDim.x - tiles);
    return;
  }
  for (int g = threadIdx.x; g < kRadixWarps * digits; g += kRadixThreads) s_at[g] = 0;
  __syncthreads();
  wait_for_previous();
  const int* count = a.count[pass];
  int* next = pass + 1 < a.passes ? a.count[pass + 1] : nullptr;
  const unsigned* key_in = a.key[(pass & 1) ^ 1];
  const int* order_in = a.order[(pass & 1) ^ 1];
  const int shift = pass * bits;
  const int64_t r0 = (int64_t)blockIdx.x * a.tile, share = a.tile / kRadixWarps;
  const int64_t w0 = r0 + warp * share, w1 = w0 + share < a.R ? w0 + share : a.R;
  int* mine = s_at + warp * digits;
  unsigned key[kRound];
  const auto take = [&](int64_t rb) {                 // the keys of the next 32 * kRound rows
#pragma unroll
    for (int u = 0; u < kRound; ++u) {
      const int64_t r = rb + 32 * u + lane;
      key[u] = r < w1 ? (FIRST ? (unsigned)a.tokens[r] : __ldcg(key_in + r)) : 0;
    }
    if (FIRST)
#pragma unroll
      for (int u = 0; u < kRound; ++u) {
        bool bad;
        key[u] = key_of(a, (int)key[u], bad);
      }
  };
  for (int64_t rb = w0; rb < w1; rb += 32 * kRound) {
    take(rb);
#pragma unroll
    for (int u = 0; u < kRound; ++u)
      if (rb + 32 * u + lane < w1) atomicAdd(&mine[key[u] >> shift & (digits - 1)], 1);
  }
  __syncthreads();
  // the first place of each (warp, digit): digits below, the same one in earlier tiles, in earlier warps;
  // a thread up to four neighbouring digits
  const int per = (digits + kRadixThreads - 1) / kRadixThreads;
  int all[4] = {}, before[4] = {}, sum = 0;
  const auto counts = [&](auto p) {
    constexpr int PER = decltype(p)::value, kTiles = kCountsAhead / PER;
    for (int t0 = 0; t0 < tiles; t0 += kTiles) {
      int c[kTiles][PER];
#pragma unroll
      for (int u = 0; u < kTiles; ++u)
#pragma unroll
        for (int q = 0; q < PER; ++q) {
          const int g = threadIdx.x * PER + q;
          c[u][q] = g < digits && t0 + u < tiles ? __ldcg(count + (size_t)(t0 + u) * digits + g) : 0;
        }
#pragma unroll
      for (int u = 0; u < kTiles; ++u)
#pragma unroll
        for (int q = 0; q < PER; ++q) {
          all[q] += c[u][q];
          if (t0 + u < (int)blockIdx.x) before[q] += c[u][q];
        }
    }
  };
  if (per == 1) counts(std::integral_constant<int, 1>());
  else if (per == 2) counts(std::integral_constant<int, 2>());
  else counts(std::integral_constant<int, 4>());
#pragma unroll
  for (int q = 0; q < 4; ++q) sum += all[q];
  int base = cta_scan(sum);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int g = threadIdx.x * per + q;
    if (q >= per || g >= digits) continue;
    int at = base + before[q];
    for (int w = 0; w < kRadixWarps; ++w) {
      const int c = s_at[w * digits + g];
      s_at[w * digits + g] = at;
      at += c;
    }
    base += all[q];
  }
  __syncthreads();
  for (int64_t rb = w0; rb < w1; rb += 32 * kRound) {
    if (share > 32 * kRound) take(rb);                // (else they are still there)
    int row[kRound];
    if (!FIRST)
#pragma unroll
      for (int u = 0; u < kRound; ++u) row[u] = rb + 32 * u + lane < w1 ? __ldcg(order_in + rb + 32 * u + lane) : 0;
#pragma unroll
    for (int u = 0; u < kRound; ++u) {                // 32 rows at a time, in order
      const int64_t r = rb + 32 * u + lane;
      const bool in = r < w1;
      const int g = in ? (int)(key[u] >> shift & (digits - 1)) : digits;
      const unsigned same = __match_any_sync(kFull, g);
      int at = 0;
      if (in) at = mine[g] + __popc(same & ((1u << lane) - 1u));
      __syncwarp();
      if (in && (same >> lane) == 1u) mine[g] = at + 1;   // the last of its digit
      __syncwarp();
      if (in) {
        a.key[pass & 1][at] = key[u];
        a.order[pass & 1][at] = FIRST ? (int)r : row[u];
        if (next) atomicAdd(next + (size_t)(at / a.tile) * digits + (key[u] >> (shift + bits) & (digits - 1)), 1);
      }
    }
  }
}

// ---- sums ------------------------------------------------------------------------------
// The ordered rows, cut into equal tiles whatever their tokens are.  A tile walks its
// rows with the columns over its threads, kBatch rows requested at once; a token's
// last row writes the sum.  A token that a border cuts leaves a piece of its sum
// (fp32) in either tile, and embed_join_kernel adds those up.  Bound by memory: 29491
// rows of d = 2048 bf16 into 12000 of the table 27 us, 6.3 TB/s.  CTAs of 128 threads
// (two a tile there): with 256 the whole gradient took 122 us instead of 115.
constexpr int kSlots = 64;                            // rows of a tile at most: two of a lane
constexpr int kBatch = 8;
constexpr int kSumThreads = 128;
// A tile's state: the token whose rows go on behind it (-1: none), and whether that one begins there or has all of
// the tile's rows and others before them.
constexpr int kThrough = 1, kBegins = 2;

template <typename T, int VE, bool ADD>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(const EmbedArgs a, int last_pass) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
  __shared__ int2 s_slot[kSlots];                     // (row or -1, token to write or -1)
  __shared__ int s_head, s_open;                      // the first rows go on from the tile before; the token left open
  const unsigned* key = a.key[last_pass & 1];
  const int* order = a.order[last_pass & 1];
  const int nvec = a.d / VE;
  wait_for_previous();
  const int tile = blockIdx.x, chunk = blockIdx.y;
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x, i0 = tile * a.slots;
    const unsigned prev = i0 > 0 ? __ldcg(key + i0 - 1) : 0xFFFFFFFFu;
    unsigned k[2], after[2];
    int row[2], n = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = i0 + lane + 32 * h;
      const bool in = i < a.R && lane + 32 * h < a.slots;
      k[h] = in ? __ldcg(key + i) : (unsigned)a.V;
      row[h] = in ? __ldcg(order + i) : 0;
      after[h] = in && i + 1 < a.R ? __ldcg(key + i + 1) : 0xFFFFFFFFu;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool in = k[h] < (unsigned)a.V;           // padding is behind all others
      s_slot[lane + 32 * h] = make_int2(in ? row[h] : -1, in && after[h] != k[h] ? (int)k[h] : -1);
      n += __popc(__ballot_sync(kFull, in));
    }
    const int tail = n - 1;                           // the last row's lane and half
    const unsigned kt = __shfl_sync(kFull, tail >= 32 ? k[1] : k[0], tail & 31);
    const unsigned at = __shfl_sync(kFull, tail >= 32 ? after[1] : after[0], tail & 31);
    if (lane == 0) {
      const bool head = n > 0 && k[0] == prev, open = n > 0 && at == kt;
      s_head = head;
      s_open = open ? (int)kt : -1;
      if (chunk == 0) a.state[tile] = make_int2(s_open, open ? (head && k[0] == kt ? kThrough : kBegins) : 0);
    }
  }
  __syncthreads();
  const int c = chunk * blockDim.x + threadIdx.x;
  if (c >= nvec) return;
  const Raw* d_x = static_cast<const Raw*>(a.d_x) + c;
  Raw* out = static_cast<Raw*>(a.d_table) + c;
  const size_t piece = (size_t)tile * a.d + (size_t)c * VE;
  float sum[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) sum[j] = 0.f;
  bool head = s_head != 0;
#pragma unroll 1
  for (int s0 = 0; s0 < a.slots; s0 += kBatch) {
    Raw x[kBatch], had[ADD ? kBatch : 1];
    int2 o[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      o[u] = s_slot[s0 + u];
      x[u] = V::zero();
      if (o[u].x >= 0) x[u] = d_x[(size_t)o[u].x * nvec];
      if (ADD && o[u].y >= 0) had[u] = out[(size_t)o[u].y * nvec];
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      float f[VE];
      V::get(x[u], f);
#pragma unroll
      for (int j = 0; j < VE; ++j) sum[j] += f[j];
      if (o[u].y >= 0) {
        if (head) {                                   // (the join writes it)
#pragma unroll
          for (int j = 0; j < VE; ++j) a.head[piece + j] = sum[j];
          head = false;
        } else {
          if (ADD) V::get(had[u], f);
#pragma unroll
          for (int j = 0; j < VE; ++j) f[j] = ADD ? __fmaf_rn(sum[j], a.scale, f[j]) : sum[j] * a.scale;
          out[(size_t)o[u].y * nvec] = V::put(f);
        }
#pragma unroll
        for (int j = 0; j < VE; ++j) sum[j] = 0.f;
      }
    }
  }
  if (s_open >= 0)
#pragma unroll
    for (int j = 0; j < VE; ++j) a.tail[piece + j] = sum[j];
}

// Tokens that borders cut: the piece of the tile where one begins, those of the
// tiles that it fills, and that of the tile where it ends, in this order.  A CTA
// kJoinTiles tiles and, with others, their columns; a warp a token and 32 JV of its
// columns, or, for a token of more than kLong tiles, the CTA's warps an eighth of the
// tiles each.  A few loads in a row: 5 us of a call; of a token that fills thousands of
// tiles many: R = 600000 d = 256 of 32000, a tenth, half, all rows of one token 146, 232,
// 342 us, with none above the others 128.
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;
constexpr int kJoinTiles = 8;
constexpr int kLong = 16;
constexpr int kPieces = 8;                            // requested at once
template <int JV>
__device__ __forceinline__ void get_piece(const float* p, float (&f)[JV]) {
  if constexpr (JV == 4) {
    const float4 v = __ldcg(reinterpret_cast<const float4*>(p));
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
  } else {
    f[0] = __ldcg(p);
  }
}
template <typename T, int JV, bool ADD>
__global__ void __launch_bounds__(kJoinThreads) embed_join_kernel(const EmbedArgs a, int tiles) {
  __shared__ int s_fills[kJoinTiles];
  __shared__ float s_sum[kJoinWarps][32][JV];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  wait_for_previous();
  const int t0 = blockIdx.x * kJoinTiles;
  const int2 st = lane < kJoinTiles && t0 + lane < tiles ? a.state[t0 + lane] : make_int2(-1, 0);
  const unsigned begins = __ballot_sync(kFull, st.y == kBegins);
  if (!begins) return;                               // (the same in every warp)
  for (int b = warp; b < kJoinTiles; b += kJoinWarps) {
    if (!(begins >> b & 1u)) continue;
    int n = 0;                                       // the tiles that the token fills
    for (;;) {
      const int t = t0 + b + 1 + n + lane;
      const unsigned through = __ballot_sync(kFull, t < tiles && a.state[t].y == kThrough);
      const int run = through == kFull ? 32 : __ffs((int)~through) - 1;
      n += run;
      if (run < 32) break;
    }
    if (lane == 0) s_fills[b] = n;
  }
  __syncthreads();
  const auto sums = [&](int first, int k0, int k1, int n, int j, float (&sum)[JV]) {   // pieces k0 .. k1 of 0 .. n + 1
#pragma unroll
    for (int q = 0; q < JV; ++q) sum[q] = 0.f;
    for (int kb = k0; kb < k1; kb += kPieces) {
      float p[kPieces][JV];
#pragma unroll
      for (int u = 0; u < kPieces; ++u)
        if (kb + u < k1) get_piece<JV>((kb + u <= n ? a.tail : a.head) + (size_t)(first + kb + u) * a.d + j, p[u]);
#pragma unroll
      for (int u = 0; u < kPieces; ++u)
#pragma unroll
        for (int q = 0; q < JV; ++q)
          if (kb + u < k1) sum[q] += p[u][q];
    }
  };
  const auto write = [&](int token, int j, const float (&sum)[JV]) {
    T* out = static_cast<T*>(a.d_table) + (size_t)token * a.d + j;
#pragma unroll
    for (int q = 0; q < JV; ++q) out[q] = from_float<T>(ADD ? __fmaf_rn(sum[q], a.scale, to_float(out[q])) : sum[q] * a.scale);
  };
  const int groups = (a.d + 32 * JV - 1) / (32 * JV), pairs = __popc(begins) * groups;
  for (int p = warp + blockIdx.y * kJoinWarps; p < pairs; p += gridDim.y * kJoinWarps) {
    unsigned left = begins;
    for (int k = p / groups; k > 0; --k) left &= left - 1;
    const int b = __ffs((int)left) - 1, n = s_fills[b];
    const int j = (p % groups * 32 + lane) * JV, token = __shfl_sync(kFull, st.x, b);
    if (n > kLong || j >= a.d) continue;
    float sum[JV];
    sums(t0 + b, 0, n + 2, n, j, sum);
    write(token, j, sum);
  }
  for (unsigned m = begins; m; m &= m - 1) {
    const int b = __ffs((int)m) - 1, n = s_fills[b], token = __shfl_sync(kFull, st.x, b);
    if (n <= kLong) continue;
    const int share = (n + 2 + kJoinWarps - 1) / kJoinWarps;
    for (int g = blockIdx.y; g < groups; g += gridDim.y) {
      const int j = (g * 32 + lane) * JV;
      float sum[JV];
      sums(t0 + b, min(warp * share, n + 2), min((warp + 1) * share, n + 2), n, min(j, a.d - JV), sum);
#pragma unroll
      for (int q = 0; q < JV; ++q) s_sum[warp][lane][q] = sum[q];
      __syncthreads();
      if (warp == 0 && j < a.d) {
#pragma unroll
        for (int q = 0; q < JV; ++q)
          for (int w = 1; w < kJoinWarps; ++w) sum[q] += s_sum[w][lane][q];
        write(token, j, sum);
      }
      __syncthreads();
    }
  }
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }
// Rows of a tile, at least kBatch, for four tiles an SM where there are few rows (for eight, 32768 rows of 1000 tokens
// took 41 us instead of 35: borders cut twice as many tokens).
// Narrow rows up to four times as many, since a tile's batches go one after another: R = 20000 of 120000, d = 256 with
// tiles of 64 31.4 us, of 16 24.9, d = 512 36.5 and (32) 32.0; eight times, d = 128 R = 32768 of 3000 24.2 against 21.4.
constexpr int kTiles = 608;
int wanted_tiles(int d) { return kTiles * std::max(1, std::min(4, 1024 / d)); }
int slot_count(int R, int d) {
  int n = kBatch;
  while (n < kSlots && R > n * wanted_tiles(d)) n *= 2;
  return n;
}
int tile_rows(int R) {
  if (R <= kShortRows) return kTileMin / 4;
  return R < 2 * kShortRows ? kTileMin / 2 : kTileMin * ceil_div(R, (int64_t)kTileMin * 256);
}
// The most tiles that R rows or fewer have, of the ordering and of the sums: a workspace that is enough for R rows is
// for fewer, although their tiles are smaller ones and may be more.
int most_tiles(int R) {
  return R <= kShortRows ? ceil_div(R, kTileMin / 4) : std::max(kShortRows / (kTileMin / 4), std::min(256, ceil_div(R, kTileMin)));
}
int most_sum_tiles(int R, int d) { return std::min(ceil_div(R, kBatch), std::max(wanted_tiles(d), ceil_div(R, kSlots))); }

}  // namespace

size_t embed_layout(EmbedArgs& a, char* w) {
  size_t o = 0;
  auto take = [&](size_t bytes) {
    char* p = w ? w + o : nullptr;
    o += up256(bytes);
    return p;
  };
  const int R = a.R > 0 ? a.R : 1;
  a.err = (unsigned*)take(sizeof(unsigned));
  int bits = 1;
  while (((int64_t)1 << bits) <= a.V) ++bits;         // keys 0 .. V
  a.passes = R <= kRankRows ? 1 : ceil_div(bits, kRadixBits);
  a.bits = ceil_div(bits, a.passes);
  a.tile = tile_rows(R);
  for (int k = 0; k < (a.passes > 1 ? 2 : 1); ++k) {
    a.key[k] = (unsigned*)take((size_t)R * 4);
    a.order[k] = (int*)take((size_t)R * 4);
  }
  if (R > kRankRows)
    for (int p = 0; p < a.passes; ++p) a.count[p] = (int*)take((size_t)most_tiles(R) << (a.bits + 2));
  a.slots = slot_count(R, a.d);
  const size_t tiles = most_sum_tiles(R, a.d);
  a.state = (int2*)take(tiles * 8);
  a.head = (float*)take(tiles * a.d * 4);
  a.tail = (float*)take(tiles * a.d * 4);
  return o;
}
cudaError_t take_embed_errors(unsigned* flags, cudaStream_t s) { return take_errors(flags, s); }

cudaError_t launch_embed(const EmbedArgs& a, cudaStream_t s) {
  return by_row_type(a.dtype, a.d, [&](auto t) {
    using Row = decltype(t);
    const int pieces = ceil_div(a.d / Row::VE, 32 * kAhead);
    const int64_t units = (int64_t)a.R * pieces;
    if constexpr (Row::VE * sizeof(typename Row::T) == 16)
      if (a.d / Row::VE <= kNarrowVecs && a.R >= kNarrowRows) {
        const int64_t ctas = ((int64_t)a.R * (a.d / Row::VE) + 256 * kAhead - 1) / (256 * kAhead);
        return launch(true, embed_narrow_kernel<typename Row::T, Row::VE>, (unsigned)(ctas < (1 << 30) ? ctas : 1 << 30), 256, 0,
                      s, a);
      }
    // a warp a CTA until every SM has some, then eight
    int warps = 1;
    while (warps < 8 && units > 304 * warps) warps *= 2;
    const int64_t ctas = (units + warps - 1) / warps;
    return launch(true, embed_kernel<typename Row::T, Row::VE>, (unsigned)(ctas < (1 << 30) ? ctas : 1 << 30), 32 * warps, 0, s, a,
                  pieces);
  });
}

namespace {
template <typename T, int VE, bool ADD>
cudaError_t launch_sums(const EmbedArgs& a, cudaStream_t s) {
  const int nvec = a.d / VE, tiles = ceil_div(a.R, a.slots);
  const int threads = nvec < kSumThreads ? (nvec + 31) / 32 * 32 : kSumThreads;
  cudaError_t e = launch(true, embed_sum_kernel<T, VE, ADD>, dim3(tiles, ceil_div(nvec, threads)), threads, 0, s, a, a.passes - 1);
  if (e != cudaSuccess) return e;
  constexpr int JV = VE * sizeof(T) == 16 ? 4 : 1;
  const int groups = ceil_div(a.d, 32 * JV);
  return launch(true, embed_join_kernel<T, JV, ADD>, dim3(ceil_div(tiles, kJoinTiles), groups < 16 ? groups : 16),
                kJoinThreads, 0, s, a, tiles);
}
}  // namespace

cudaError_t launch_embed_backward(const EmbedArgs& args, cudaStream_t s) {
  EmbedArgs a = args;
  if (a.R <= kFewRows)
    return by_row_type(a.dtype, a.d, [&](auto t) {
      using Row = decltype(t);
      return a.add ? launch_few<typename Row::T, Row::VE, true>(a, s) : launch_few<typename Row::T, Row::VE, false>(a, s);
    });
  // the k-th of the launches that order the rows fills bytes [fill[k], fill[k + 1])
  const size_t all = a.add ? 0 : (size_t)a.V * a.d * (a.dtype == 0 ? 4 : 2);
  const int launches = a.R <= kRankRows ? 1 : a.passes + 1;
  for (int k = 0; k < launches; ++k) a.fill[k] = all / launches / 16 * 16 * k;
  a.fill[launches] = all;
  const auto fill_ctas = [&](int k) { return (int)std::min((a.fill[k + 1] - a.fill[k] + kFillChunk - 1) / kFillChunk, kFillCtas); };
  cudaError_t e;
  if (a.R <= kRankRows) {
    const size_t smem = (size_t)(a.R + 127) / 128 * 512;
    const int per = a.R <= 1216 ? 8 : 32, ctas = ceil_div(a.R, per);
    // (of many rows it is bound by the SMs' instructions, and CTAs that come early crowd on a few of them: R = 4096 d = 512
    // added to 18.3 us a call in a row of them instead of 10.2, written whole, 33 MB, 16.4 and 13.6; behind zeros that take
    // longer nobody waits for them.  Early and not, d = 1024, MB of zeros: R = 2500 48 15.8 and 14.9, 64 16.8 and 17.1; R =
    // 4096 64 19.8 and 19.3, 96 23.6 and 24.0, 256 45.0 and 45.6; R = 7168 64 29.8 and 22.7, 96 30.3 and 27.7, 128 31.5
    // and 32.3)
    const bool early = per == 8 || all >= std::max(kManyZeros, a.R * kManyZerosRow);
    e = launch(early, per == 8 ? embed_rank_kernel<1> : embed_rank_kernel<4>, ctas + fill_ctas(0), kRankThreads, smem, s, a, ctas);
  } else {
    const int digits = 1 << a.bits, tiles = ceil_div(a.R, a.tile);
    const size_t smem = (size_t)kRadixWarps * digits * 4;
    e = launch(true, embed_count_kernel, tiles + fill_ctas(0), kRadixThreads, (size_t)digits * 4, s, a, digits, tiles);
    for (int p = 0; p < a.passes && e == cudaSuccess; ++p)
      e = launch(true, p == 0 ? embed_move_kernel<true> : embed_move_kernel<false>, tiles + fill_ctas(p + 1), kRadixThreads, smem,
                 s, a, p, a.bits, tiles);
  }
  if (e != cudaSuccess) return e;
  return by_row_type(a.dtype, a.d, [&](auto t) {
    using Row = decltype(t);
    return a.add ? launch_sums<typename Row::T, Row::VE, true>(a, s) : launch_sums<typename Row::T, Row::VE, false>(a, s);
  });
}

}  // namespace cmsd
