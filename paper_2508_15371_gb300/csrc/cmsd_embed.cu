// Scaled rows of the token table (include/cmsd.h, cmsd_embedding) and the
// table's gradient (cmsd_embedding_backward).
//
// The gradient's rows are put into the order of their tokens first (stable: rows
// of one token keep theirs), by tokens alone; then every row of d_x is read and
// every row of d_table written once.
#include <cuda_bf16.h>

#include "cmsd_device.cuh"
#include "cmsd_errors.cuh"
#include "cmsd_launch.cuh"
#include "cmsd_rows.cuh"
#include "cmsd_train.h"

namespace cmsd {
namespace {

__device__ __forceinline__ void wait_for_previous() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ---- rows of the table ------------------------------------------------------------
// A warp a piece of 256 vectors of a row, eight requested at once.
constexpr int kAhead = 8;
template <typename T, int VE>
__global__ void __launch_bounds__(256) embed_kernel(const EmbedArgs a, int pieces) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
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
      if (keep && v0 + 32 * k < nvec) w[k] = __ldg(row + v0 + 32 * k);
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

// ---- the rows in their tokens' order ------------------------------------------------
// What a row is ordered by: its token, or V (behind all tokens) for padding.
__device__ __forceinline__ unsigned key_of(const EmbedArgs& a, int token, bool& bad) {
  const bool in = token >= 0 && token < a.V;
  bad = !in && token != a.ignore;
  return in && token != a.ignore ? (unsigned)token : (unsigned)a.V;
}

// Few rows: each row's place is the number of rows before it in (token, row)
// order, counted by comparing it with all of them: R^2 comparisons, spread over
// the GPU, in one launch.  A warp RPW rows, a lane every 32nd four of the others.
constexpr int kRankRows = 8192;
constexpr int kRankThreads = 256;
template <int RPW>
__global__ void __launch_bounds__(kRankThreads) embed_rank_kernel(const EmbedArgs a) {
  extern __shared__ uint4 s_key4[];
  unsigned* s_key = reinterpret_cast<unsigned*>(s_key4);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, padded = (a.R + 127) / 128 * 128;
  for (int r = threadIdx.x; r < padded; r += kRankThreads) {
    bool bad = false;
    unsigned k = 0xFFFFFFFFu;
    if (r < a.R) {
      k = key_of(a, a.tokens[r], bad);
      if (bad && blockIdx.x == 0) report(a.err, 1u);
    }
    s_key[r] = k;
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
  // rows before: not above; rows behind: below
  const int own = r0 / 128, all = padded / 128;
#pragma unroll 4
  for (int c = 0; c < own; ++c) {
    const uint4 t = s_key4[c * 32 + lane];
#pragma unroll
    for (int j = 0; j < RPW; ++j) n[j] += (t.x <= key[j]) + (t.y <= key[j]) + (t.z <= key[j]) + (t.w <= key[j]);
  }
#pragma unroll 4
  for (int c = own + 1; c < all; ++c) {
    const uint4 t = s_key4[c * 32 + lane];
#pragma unroll
    for (int j = 0; j < RPW; ++j) n[j] += (t.x < key[j]) + (t.y < key[j]) + (t.z < key[j]) + (t.w < key[j]);
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
constexpr int kRadixBits = 10;
constexpr int kRadixThreads = 256, kRadixWarps = kRadixThreads / 32;
constexpr int kTileMin = 2048;
__global__ void __launch_bounds__(kRadixThreads) embed_count_kernel(const EmbedArgs a, int digits) {
  extern __shared__ int s_count[];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int g = threadIdx.x; g < digits; g += kRadixThreads) s_count[g] = 0;
  __syncthreads();
  const int64_t r0 = (int64_t)blockIdx.x * a.tile, r1 = r0 + a.tile < a.R ? r0 + a.tile : a.R;
  for (int64_t r = r0 + threadIdx.x; r < r1; r += kRadixThreads) {
    bool bad;
    const unsigned k = key_of(a, a.tokens[r], bad);
    if (bad) report(a.err, 1u);
    atomicAdd(&s_count[k & (digits - 1)], 1);
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
__global__ void __launch_bounds__(kRadixThreads) embed_move_kernel(const EmbedArgs a, int pass, int bits) {
  extern __shared__ int s_at[];                       // [kRadixWarps][digits]: counts, then the next place of each
  const int digits = 1 << bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tiles = gridDim.x;
  wait_for_previous();
  const int* count = a.count[pass];
  int* next = pass + 1 < a.passes ? a.count[pass + 1] : nullptr;
  const unsigned* key_in = a.key[(pass & 1) ^ 1];
  const int* order_in = a.order[(pass & 1) ^ 1];
  const int shift = pass * bits;
  for (int g = threadIdx.x; g < kRadixWarps * digits; g += kRadixThreads) s_at[g] = 0;
  __syncthreads();
  const int64_t r0 = (int64_t)blockIdx.x * a.tile, share = a.tile / kRadixWarps;
  const int64_t w0 = r0 + warp * share, w1 = w0 + share < a.R ? w0 + share : a.R;
  int* mine = s_at + warp * digits;
  for (int64_t r = w0 + lane; r < w1; r += 32) {
    bool bad;
    const unsigned k = FIRST ? key_of(a, a.tokens[r], bad) : key_in[r];
    atomicAdd(&mine[k >> shift & (digits - 1)], 1);
  }
  __syncthreads();
  // the first place of each (warp, digit): digits below, the same one in earlier tiles, in earlier warps;
  // a thread up to four neighbouring digits
  const int per = (digits + kRadixThreads - 1) / kRadixThreads;
  int all[4], before[4], sum = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    all[q] = before[q] = 0;
    const int g = threadIdx.x * per + q;
    if (q >= per || g >= digits) continue;
    int b = 0, rest = 0;
#pragma unroll 8
    for (int t = 0; t < tiles; ++t) {
      const int c = __ldcg(count + (size_t)t * digits + g);
      if (t < (int)blockIdx.x) b += c;
      else rest += c;
    }
    before[q] = b;
    all[q] = b + rest;
    sum += all[q];
  }
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
  for (int64_t rb = w0; rb < w1; rb += 32) {          // 32 rows at a time, in order
    const int64_t r = rb + lane;
    const bool in = r < w1;
    unsigned k = 0;
    int row = (int)r;
    if (in) {
      bool bad;
      k = FIRST ? key_of(a, a.tokens[r], bad) : key_in[r];
      if (!FIRST) row = order_in[r];
    }
    const int g = in ? (int)(k >> shift & (digits - 1)) : digits;
    const unsigned same = __match_any_sync(kFull, g);
    int at = 0;
    if (in) at = mine[g] + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (in && (same >> lane) == 1u) mine[g] = at + 1;   // the last of its digit
    __syncwarp();
    if (in) {
      a.key[pass & 1][at] = k;
      a.order[pass & 1][at] = row;
      if (next) atomicAdd(next + (size_t)(at / a.tile) * digits + (k >> (shift + bits) & (digits - 1)), 1);
    }
  }
}

// ---- sums ------------------------------------------------------------------------------
// The work is a list of slots, cut into equal tiles whatever the tokens are.
// Written whole: token v has a slot for each of its rows and one more, so row i of
// the ordered ones is slot key_i + i, and the slot after a token's rows writes
// zeros where it had none.  Added to: row i is slot i.  A tile walks its slots with
// the columns over its threads, kBatch rows requested at once; a token's last row
// writes the sum.  A token that a border cuts leaves a piece of its sum (fp32) in
// either tile, and embed_join_kernel adds those up.  Bound by memory.
constexpr int kSlots = 64;                            // slots of a tile
constexpr int kBatch = 8;
constexpr int kSumThreads = 256;

template <bool ADD>
__device__ __forceinline__ int64_t slot_of(const EmbedArgs& a, int64_t i, unsigned key) {
  return ADD ? i : i + (int64_t)key;
}
// the first ordered row whose slot is not below `slot`, by a warp
__device__ __forceinline__ int64_t first_row(const EmbedArgs& a, const unsigned* key, int64_t slot) {
  int64_t lo = 0, hi = a.R;                           // it is in [lo, hi]
  while (hi > lo) {
    const int64_t step = (hi - lo + 31) / 32, i = lo + (threadIdx.x & 31) * step;
    const bool below = i < hi && i + (int64_t)__ldcg(key + i) < slot;
    const int n = __popc(__ballot_sync(kFull, below));
    if (n == 0) return lo;
    const int64_t last = lo + (n - 1) * step;         // the last probe below
    hi = last + step < hi ? last + step : hi;
    lo = last + 1;
  }
  return lo;
}

// A tile's state: the token whose rows go on behind it (-1: none), whether that one begins there or has all of the
// tile's rows and others before them, and the place of the tile's pieces.
constexpr int kThrough = 1, kBegins = 2;

template <typename T, int VE, bool ADD>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(const EmbedArgs a, int last_pass) {
  using V = RowVec<T, VE>;
  using Raw = typename V::Raw;
  __shared__ int2 s_slot[kSlots];                     // (row or -1, token to write or -1)
  __shared__ int s_head, s_open, s_piece;             // the first rows go on from the tile before; the token left open
  const unsigned* key = a.key[last_pass & 1];
  const int* order = a.order[last_pass & 1];
  const int64_t slot0 = (int64_t)blockIdx.x * kSlots;
  wait_for_previous();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    const int64_t i0 = ADD ? slot0 : first_row(a, key, slot0);
    // the rows of the tile, at most one a slot
    const unsigned prev = i0 > 0 ? __ldcg(key + i0 - 1) : 0xFFFFFFFFu;
    unsigned k[2], after[2];
    int q[2];
    unsigned rows[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t i = i0 + lane + 32 * h;
      k[h] = i < a.R ? __ldcg(key + i) : (unsigned)a.V;
      after[h] = i + 1 < a.R ? __ldcg(key + i + 1) : 0xFFFFFFFFu;
      const int64_t s = slot_of<ADD>(a, i, k[h]) - slot0;
      q[h] = k[h] < (unsigned)a.V && s < kSlots ? (int)s : -1;
      if (q[h] >= 0) rows[q[h] >> 5] |= 1u << (q[h] & 31);
    }
    rows[0] = __reduce_or_sync(kFull, rows[0]);
    rows[1] = __reduce_or_sync(kFull, rows[1]);
    const int n = __popc(rows[0]) + __popc(rows[1]);
    // slots without a row: zeros, where the token has none
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int s = lane + 32 * h;
      if (!(rows[h] >> lane & 1u)) {
        const int before = (h ? __popc(rows[0]) : 0) + __popc(rows[h] & ((1u << lane) - 1u));
        const int64_t v = slot0 + s - i0 - before;
        int2 o = make_int2(-1, -1);
        if (!ADD && v < a.V) {
          const unsigned p = before > 0 ? __ldcg(key + i0 + before - 1) : prev;
          if (p != (unsigned)v) o.y = (int)v;
        }
        s_slot[s] = o;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (q[h] >= 0)
        s_slot[q[h]] = make_int2(order[i0 + lane + 32 * h], after[h] != k[h] ? (int)k[h] : -1);
    const int tail = n - 1;                           // the last row's lane and half
    const unsigned kt = __shfl_sync(kFull, tail >= 32 ? k[1] : k[0], tail & 31);
    const unsigned at = __shfl_sync(kFull, tail >= 32 ? after[1] : after[0], tail & 31);
    const unsigned kf = __shfl_sync(kFull, k[0], 0);
    if (lane == 0) {
      const bool head = n > 0 && kf == prev, open = n > 0 && at == kt;
      s_head = head;
      s_open = open ? (int)kt : -1;
      // (places by the first row where there are fewer rows than tiles)
      s_piece = a.pieces == a.R ? (int)i0 : (int)blockIdx.x;
      if (blockIdx.y == 0)
        a.state[blockIdx.x] = make_int4(s_open, open ? (head && kf == kt ? kThrough : kBegins) : 0, s_piece, 0);
    }
  }
  __syncthreads();
  const int nvec = a.d / VE, c = blockIdx.y * blockDim.x + threadIdx.x;
  if (c >= nvec) return;
  const Raw* d_x = static_cast<const Raw*>(a.d_x) + c;
  Raw* out = static_cast<Raw*>(a.d_table) + c;
  const size_t piece = (size_t)s_piece * a.d + (size_t)c * VE;
  float sum[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) sum[j] = 0.f;
  bool head = s_head != 0;
#pragma unroll 1
  for (int s0 = 0; s0 < kSlots; s0 += kBatch) {
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
      if (o[u].x >= 0) {
        float f[VE];
        V::get(x[u], f);
#pragma unroll
        for (int j = 0; j < VE; ++j) sum[j] += f[j];
      }
      if (o[u].y >= 0) {
        if (o[u].x >= 0 && head) {                    // (the join writes it)
#pragma unroll
          for (int j = 0; j < VE; ++j) a.head[piece + j] = sum[j];
          head = false;
        } else {
          float f[VE];
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
// tiles that it fills, and that of the tile where it ends, in this order.  A CTA 32
// tiles; a warp a token and 32 of its columns.
constexpr int kJoinThreads = 256;
template <typename T, bool ADD>
__global__ void __launch_bounds__(kJoinThreads) embed_join_kernel(const EmbedArgs a, int tiles) {
  const int lane = threadIdx.x & 31;
  wait_for_previous();
  const int t0 = blockIdx.x * 32;
  const int4 st = t0 + lane < tiles ? a.state[t0 + lane] : make_int4(-1, 0, 0, 0);
  const unsigned begins = __ballot_sync(kFull, st.y == kBegins);
  const int groups = (a.d + 31) / 32, pairs = __popc(begins) * groups;
  for (int p = (threadIdx.x >> 5) + blockIdx.y * (kJoinThreads / 32); p < pairs; p += gridDim.y * (kJoinThreads / 32)) {
    const int b = __fns(begins, 0, p / groups + 1);
    const int j = p % groups * 32 + lane, token = __shfl_sync(kFull, st.x, b);
    const int place = __shfl_sync(kFull, st.z, b);
    const int first = t0 + b;
    // the tiles that the token fills
    int n = 0;
    for (;;) {
      const int t = first + 1 + n + lane;
      const unsigned through = __ballot_sync(kFull, t < tiles && a.state[t].y == kThrough);
      const int run = through == kFull ? 32 : __ffs(~through) - 1;
      n += run;
      if (run < 32) break;
    }
    if (j >= a.d) continue;
    float sum = __ldcg(a.tail + (size_t)place * a.d + j);
#pragma unroll 8
    for (int k = 1; k <= n; ++k) sum += __ldcg(a.tail + (size_t)a.state[first + k].z * a.d + j);
    sum += __ldcg(a.head + (size_t)a.state[first + n + 1].z * a.d + j);
    T* out = static_cast<T*>(a.d_table) + (size_t)token * a.d + j;
    *out = from_float<T>(ADD ? __fmaf_rn(sum, a.scale, to_float(*out)) : sum * a.scale);
  }
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

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
  a.tile = kTileMin * ceil_div(R, (int64_t)kTileMin * 256);
  for (int k = 0; k < (a.passes > 1 ? 2 : 1); ++k) {
    a.key[k] = (unsigned*)take((size_t)R * 4);
    a.order[k] = (int*)take((size_t)R * 4);
  }
  if (R > kRankRows)
    for (int p = 0; p < a.passes; ++p) a.count[p] = (int*)take((size_t)ceil_div(R, a.tile) << (a.bits + 2));
  const int tiles = ceil_div((int64_t)a.V + R, kSlots);
  a.pieces = R < tiles ? R : tiles;
  a.state = (int4*)take((size_t)tiles * 16);
  a.head = (float*)take((size_t)a.pieces * a.d * 4);
  a.tail = (float*)take((size_t)a.pieces * a.d * 4);
  return o;
}
cudaError_t take_embed_errors(unsigned* flags, cudaStream_t s) { return take_errors(flags, s); }

cudaError_t launch_embed(const EmbedArgs& a, cudaStream_t s) {
  return by_row_type(a.dtype, a.d, [&](auto t) {
    using Row = decltype(t);
    const int pieces = ceil_div(a.d / Row::VE, 32 * kAhead);
    const int64_t units = (int64_t)a.R * pieces;
    // a warp a CTA until every SM has some, then eight
    int warps = 1;
    while (warps < 8 && units > 304 * warps) warps *= 2;
    const int64_t ctas = (units + warps - 1) / warps;
    embed_kernel<typename Row::T, Row::VE><<<(unsigned)(ctas < (1 << 30) ? ctas : 1 << 30), 32 * warps, 0, s>>>(a, pieces);
    return cudaGetLastError();
  });
}

namespace {
template <typename T, int VE, bool ADD>
cudaError_t launch_sums(const EmbedArgs& a, cudaStream_t s) {
  const int nvec = a.d / VE, tiles = ceil_div(ADD ? (int64_t)a.R : (int64_t)a.V + a.R, kSlots);
  const int threads = nvec < kSumThreads ? (nvec + 31) / 32 * 32 : kSumThreads;
  cudaError_t e = launch(true, embed_sum_kernel<T, VE, ADD>, dim3(tiles, ceil_div(nvec, threads)), threads, 0, s, a,
                         a.passes - 1);
  if (e != cudaSuccess) return e;
  const int groups = ceil_div(a.d, 32);
  return launch(true, embed_join_kernel<T, ADD>, dim3(ceil_div(tiles, 32), groups < 8 ? 1 : 4), kJoinThreads, 0, s, a, tiles);
}
}  // namespace

cudaError_t launch_embed_backward(const EmbedArgs& a, cudaStream_t s) {
  cudaError_t e;
  if (a.R <= kRankRows) {
    const size_t smem = (size_t)(a.R + 127) / 128 * 512;
    if (a.R <= 2432) e = launch(false, embed_rank_kernel<1>, ceil_div(a.R, 8), kRankThreads, smem, s, a);
    else e = launch(false, embed_rank_kernel<4>, ceil_div(a.R, 32), kRankThreads, smem, s, a);
  } else {
    const int digits = 1 << a.bits, tiles = ceil_div(a.R, a.tile);
    const size_t smem = (size_t)kRadixWarps * digits * 4;
    e = launch(false, embed_count_kernel, tiles, kRadixThreads, (size_t)digits * 4, s, a, digits);
    for (int p = 0; p < a.passes && e == cudaSuccess; ++p)
      e = p == 0 ? launch(true, embed_move_kernel<true>, tiles, kRadixThreads, smem, s, a, p, a.bits)
                 : launch(true, embed_move_kernel<false>, tiles, kRadixThreads, smem, s, a, p, a.bits);
  }
  if (e != cudaSuccess) return e;
  return by_row_type(a.dtype, a.d, [&](auto t) {
    using Row = decltype(t);
    return a.add ? launch_sums<typename Row::T, Row::VE, true>(a, s) : launch_sums<typename Row::T, Row::VE, false>(a, s);
  });
}

}  // namespace cmsd
