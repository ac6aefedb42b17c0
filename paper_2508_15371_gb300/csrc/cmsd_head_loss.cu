// The head's loss and its gradients (include/cmsd.h, cmsd_lmhead_loss and
// cmsd_lmhead_loss_backward).
//
// Forward: the logits of a tile of rows and vocabulary entries are formed in
// tensor memory and reduced at once to each row's maximum and sum of exponentials
// over the tile's entries; a second kernel merges a row's tiles.  Backward, a
// piece of the vocabulary at a time: the logits again, from them the piece of
// P (bf16), then P W, summed over the pieces in fp32, and P^T h.
#include <cuda_bf16.h>

#include "cmsd_head.h"
#include "cmsd_tc.cuh"

namespace cmsd {
namespace {

__device__ __forceinline__ bool kept(const HeadLossArgs& a, int label) {
  return label != a.ignore && label >= 0 && label < a.V;
}

// ---- the kept rows, packed --------------------------------------------------------
constexpr int kPackThreads = 256;
constexpr int kPackWarps = kPackThreads / 32;
constexpr int kPackZero = 8;                         // CTAs that fill rows behind the last with zeros
// kept rows among labels [0, r), the whole CTA's answer
__device__ __forceinline__ int count_kept(const HeadLossArgs& a, int r) {
  __shared__ int s_sum[kPackWarps];
  int c = 0;
  for (int k = threadIdx.x; k < r; k += kPackThreads) c += kept(a, a.labels[k]);
  c = __reduce_add_sync(kFull, c);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = c;
  __syncthreads();
  c = 0;
#pragma unroll
  for (int w = 0; w < kPackWarps; ++w) c += s_sum[w];
  return c;
}
// Each CTA packs `rows` consecutive rows: it counts the kept rows before its
// own in the labels (a prefix of them, read again by every CTA), then copies,
// a warp a row.  The last kPackZero CTAs count them all and fill up to the next
// multiple of 64 rows, the step of d_weight's sum, with zeros.
__global__ void __launch_bounds__(kPackThreads) head_pack_kernel(const HeadLossArgs a, int rows, int row_ctas) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if ((int)blockIdx.x >= row_ctas) {
    const int z = blockIdx.x - row_ctas, n = count_kept(a, a.R);
    const int end = max(1, (n + 63) / 64) * 64;
    if (z == 0 && tid == 0) *a.n = n;
    for (int p = n + z * kPackWarps + warp; p < end; p += kPackZero * kPackWarps) {
      uint4* dst = reinterpret_cast<uint4*>(a.packed + (size_t)p * a.d);
      for (int j = lane; j < a.d / 8; j += 32) dst[j] = make_uint4(0, 0, 0, 0);
    }
    return;
  }
  const int r0 = blockIdx.x * rows, r1 = min(a.R, r0 + rows);
  // a warp's first row is requested before its place is known
  constexpr int kAhead = 8;
  const int vecs = a.d / 8;
  uint4 v[kAhead];
  const uint4* ahead = reinterpret_cast<const uint4*>(a.hidden + (size_t)min(r0 + warp, a.R - 1) * a.d);
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (lane + 32 * u < vecs) v[u] = ahead[lane + 32 * u];
  int base = count_kept(a, r0);
  for (int r = r0; r < r1; r += kPackWarps) {
    // every warp knows the places of the group's rows
    const int mine = r + lane;
    const bool in = lane < kPackWarps && mine < r1;
    const int label = in ? a.labels[mine] : a.ignore;
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
        report(a.err, 1u);
      }
    }
    const int row = r + warp;
    if (row < r1 && ((k >> warp) & 1u)) {
      const int p = base + __popc(k & ((1u << warp) - 1u));
      const uint4* src = reinterpret_cast<const uint4*>(a.hidden + (size_t)row * a.d);
      uint4* dst = reinterpret_cast<uint4*>(a.packed + (size_t)p * a.d);
      int j = lane;
      if (r == r0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u, j += 32)
          if (j < vecs) dst[j] = v[u];
      }
#pragma unroll 4
      for (; j < vecs; j += 32) dst[j] = src[j];
    }
    base += __popc(k);
  }
}

// (maximum, sum) of two sets of entries, in base 2; an empty set is (-inf, 0), and
// a NaN in either sum stays
__device__ __forceinline__ void fold(float& m, float& s, float m2, float s2) {
  const float mm = fmaxf(m, m2);
  s = (s != 0.f ? s * ex2(m - mm) : 0.f) + (s2 != 0.f ? s2 * ex2(m2 - mm) : 0.f);
  m = mm;
}

// ---- the products -------------------------------------------------------------------
//
// Three products of one shape: 256 x 256 outputs of a pair of CTAs
// (tcgen05.mma, cta_group::2: each CTA holds 128 rows of A, 128 of B's 256
// columns' rows, and 128 rows of the accumulator), summed over K in steps of
// 64.  A pair reads (256 + 256) * 2 bytes of its operands per K from L2 for
// 256 * 256 products; one CTA alone with a 128 x 256 tile would read half as
// much again per product, and L2 would bound the tensor cores.  (R=4096 d=2048
// V=128256, 2867 rows kept, a few calls in a graph: loss 855-885 us, 1.70-1.76
// PFLOP/s; both gradients 2680-2800 us, 1.61-1.69.  Back to back, under the power
// limit: 964-998 us, 1.51-1.56; 2970-3097 us, 1.46-1.52.  Counters at R=2048 d=2048
// V=65536: loss 80 % of the tensor pipe, 15 TB/s from L2; gradients 80 %; P 72 %.)
//   logits   A = packed rows, B = weight, K = d; both rows of 128 bytes along K
//   d_hidden A = P, B = weight (its rows run along N), K = the piece's entries
//   d_weight A = P (its rows run along M), B = packed rows (along N), K = rows
// (kOpFewGrad, with few rows: d_hidden has A = weight (along M = d), B = P, N the
// rows.)
// One pair runs through its share of the tiles, which are dealt out ahead:
//   warp 0      lane 0 fills the ring of stages (TMA), each CTA its own halves,
//               counted at the first CTA's barrier;
//   warp 1      lane 0 of the first CTA issues the MMAs of both;
//   warps 2..9  the epilogue: warp w reads TMEM lanes 32 (w mod 4) .., the two
//               warps of a quarter 128 of the 256 columns each (the logits: warps
//               2..17, 64 columns each, whose sums stay in registers).
// Barriers: full (TMA -> MMA), empty (MMA -> TMA, in both CTAs), tfull (MMA ->
// epilogue, in both) and tempty (both epilogues -> MMA) for each of the two
// accumulators.  Every wait is bounded.
enum Op { kOpStats, kOpDz, kOpGrad, kOpFewGrad };
__host__ __device__ constexpr bool grad_op(int op) { return op == kOpGrad || op == kOpFewGrad; }
constexpr int kPairTile = kHeadTile;
constexpr int kStages = 6;
constexpr int kHalfBytes = 128 * 128;                 // 128 rows of 64 bf16
constexpr int kStageBytes = 2 * kHalfBytes;           // A's and B's half
constexpr int kEpiWarps = 8;
__host__ __device__ constexpr int epi_warps(int op) { return grad_op(op) ? kEpiWarps : 16; }
constexpr int kPairThreads = 64 + 32 * kEpiWarps;
constexpr int kOutBytes = 32 * 128;                   // a warp's 32 rows of 128 bytes on their way out
constexpr int kDzBytes = 32 * 64;                     // a warp's 32 rows of 32 entries of P
static_assert(16 * kDzBytes <= kEpiWarps * kOutBytes, "P's buffers");
constexpr size_t kPairSmem = 1024 + (size_t)kStages * kStageBytes + (size_t)kEpiWarps * kOutBytes + 8 * (2 * kStages + 4) + 16;
constexpr int kTmemCols = 512;
// The tensor cores round their sums towards zero at each step of 16 of K: at
// d=2048 logits came out short by 1.5e-6 of their size, all in the same direction,
// and losses wrong by 1.1e-6.  So the logits' sums are cut after kSumBlocks blocks of
// 64 and added up in registers: each part is shorter and smaller (losses 4.5e-7 to
// 5.9e-7 for d from 1024 to 2^20; parts of 8 blocks 2.6e-7, but 914 against 880 us at
// R=4096 d=2048 V=128256, 857 uncut).  P is formed from sums cut alike: its logits are then those
// of the lse that it is given, to the bit, and p - 1 of a label with nearly all of
// the probability is right although both are off by more than it is.
constexpr int kSumBlocks = 16;
static_assert(kPairSmem <= 227 * 1024, "shared memory");

// One tile of a pair: rows and columns of 256, K from k0 in blocks of 64.
struct Tile {
  int m, n;              // tile indices
  int k0, kb;            // first block of 64 of K and their number
  bool dw;               // kOpGrad: d_weight's product
  int part;              // kOpGrad: part of d_hidden's K
};
struct Work {
  int pairs, pair;
  int mt, nt;            // kOpStats, kOpDz: tiles of rows and of the vocabulary; kOpGrad: of rows and of d
  int total;             // tiles of this pair
  int kd;                // blocks of K of the logits, or of a part of d_hidden
  int kall;              // blocks of the whole piece (kOpGrad)
  int kw;                // blocks of K of d_weight
  int nh, mine_h;        // tiles of d_hidden, and this pair's
  int lead, boost, first, stride;   // d_weight: see below
};

// Tiles of the logits go round the pairs with the rows first, so that pairs
// running together share the weight's tile and the packed rows.  Tiles of
// d_hidden, the longer ones, go round first; pairs with one of them less then
// take `boost` tiles of d_weight more, and the rest goes round.  With few rows
// d_hidden's tiles read the weight and d_weight's are all writing, so every second
// pair runs through its tiles from the end.
template <int OP>
__device__ __forceinline__ Work work_of(const HeadLossArgs& a, int n, int vlen, bool want_h, bool want_w) {
  Work w;
  w.pairs = gridDim.x / 2;
  w.pair = blockIdx.x / 2;
  const int rows = OP == kOpFewGrad ? 1 : max(1, (n + kPairTile - 1) / kPairTile);
  if (!grad_op(OP)) {
    w.mt = rows;
    w.nt = (vlen + kPairTile - 1) / kPairTile;
    w.kd = (a.d + 63) / 64;
    const int all = w.mt * w.nt;
    w.total = all > w.pair ? (all - w.pair + w.pairs - 1) / w.pairs : 0;
    return w;
  }
  w.mt = rows;
  w.nt = (a.d + kPairTile - 1) / kPairTile;
  w.kall = (vlen + 63) / 64;
  w.kd = (w.kall + a.split - 1) / a.split;
  w.kw = max(1, (n + 63) / 64);
  w.nh = want_h ? w.mt * w.nt * a.split : 0;
  const int nw = want_w ? (vlen + kPairTile - 1) / kPairTile * w.nt : 0;
  const int rem = w.nh % w.pairs;                  // pairs [0, rem) have one tile of d_hidden more
  w.mine_h = w.nh / w.pairs + (w.pair < rem ? 1 : 0);
  w.lead = rem > 0 && w.pair >= rem ? w.pairs - rem : 0;      // this pair catches up with so many others
  const int behind = rem > 0 ? w.pairs - rem : 0;
  const int cost = OP == kOpFewGrad ? w.kw + 4 : w.kw;        // of a tile of d_weight, with few rows its writing
  int boost = behind > 0 ? (w.kd + cost / 2) / cost : 0;
  if ((long long)boost * behind > nw) boost = behind > 0 ? (nw + behind - 1) / behind : 0;
  const int early = min(nw, boost * behind);
  w.boost = 0;
  if (w.lead > 0) {
    const int at = w.pair - rem;
    w.boost = early > at ? (early - at + behind - 1) / behind : 0;
  }
  // the rest goes round, beginning behind the early ones
  const int turn = behind > 0 ? (w.pair - rem + w.pairs) % w.pairs : w.pair;
  w.first = early + turn;
  w.stride = w.pairs;
  const int late = nw > w.first ? (nw - w.first + w.pairs - 1) / w.pairs : 0;
  w.total = w.mine_h + w.boost + late;
  if (w.lead > 0) w.lead = w.pair - rem;           // index of the first early tile
  return w;
}
template <int OP>
__device__ __forceinline__ Tile tile_of(const HeadLossArgs& a, const Work& w, int i) {
  Tile t;
  if (OP == kOpFewGrad && (w.pair & 1)) i = w.total - 1 - i;
  t.dw = false;
  t.part = 0;
  t.k0 = 0;
  if (!grad_op(OP)) {
    const int j = w.pair + i * w.pairs;
    t.n = j / w.mt;
    t.m = j - t.n * w.mt;
    t.kb = w.kd;
    return t;
  }
  if (i < w.mine_h) {
    const int j = w.pair + i * w.pairs;
    const int per = w.mt * w.nt;
    t.part = j / per;
    const int r = j - t.part * per;
    t.m = r / w.nt;
    t.n = r - t.m * w.nt;
    t.k0 = t.part * w.kd;
    t.kb = max(0, min(w.kd, w.kall - t.k0));
    return t;
  }
  i -= w.mine_h;
  const int behind_early = i < w.boost ? w.lead + i * (w.pairs - w.nh % w.pairs) : w.first + (i - w.boost) * w.stride;
  t.dw = true;
  t.m = behind_early / w.nt;                       // tile of the vocabulary
  t.n = behind_early - t.m * w.nt;
  t.kb = w.kw;
  return t;
}

struct Maps {
  CUtensorMap rows_k;      // packed rows in boxes of 64 (d) x 128 rows
  CUtensorMap rows_n;      // packed rows in boxes of 64 (d) x 64 rows
  CUtensorMap weight_k;    // weight, 64 (d) x 128 entries
  CUtensorMap weight_n;    // weight, 64 (d) x 64 entries
  CUtensorMap dz_k;        // P, 64 (entries) x 128 rows
  CUtensorMap dz_m;        // P, 64 (entries) x 64 rows
  CUtensorMap dz_out;      // P, 32 (entries) x 32 rows
  CUtensorMap dw_out;      // d_weight, 64 (d) x 32 entries
  CUtensorMap dh_out;      // d_hidden's parts, 32 (d) x 32 rows
};

__device__ __forceinline__ uint32_t pack_bf(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// v0, vlen: the piece of the vocabulary; first: the first piece; cols: kOpFewGrad's
// rows, a multiple of 32
template <int OP>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(64 + 32 * epi_warps(OP), 1)
    head_pair_kernel(const HeadLossArgs a, const int v0, const int vlen, const int first, const int cols,
                     const __grid_constant__ Maps maps) {
  extern __shared__ __align__(1024) unsigned char pair_smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_rank();
  const uint32_t raw = smem_addr(pair_smem);
  const uint32_t base = (raw + 1023u) & ~1023u;
  const uint32_t bars = base + kStages * kStageBytes + kEpiWarps * kOutBytes;
  const uint32_t full = bars, empty = bars + 8 * kStages, tfull = bars + 16 * kStages, tempty = tfull + 16;
  uint32_t* s_taddr = reinterpret_cast<uint32_t*>(pair_smem + (bars - raw) + 8 * (2 * kStages + 4));
  if (tid == 0) {
    for (int k = 0; k < kStages; ++k) {
      mbar_init(full + 8 * k, 1);
      mbar_init(empty + 8 * k, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(tfull + 8 * b, 1);
      mbar_init(tempty + 8 * b, 2 * epi_warps(OP));
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(s_taddr)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tmem_fence_before();
  cluster_sync_all();
  tmem_fence_after();
  const uint32_t tbase = *s_taddr;
  bool ok = true;
  // Everything up to its griddepcontrol.wait, in each warp that waits for it
  // below, overlaps the end of what precedes this grid on the stream.
  Work w0;                                           // of one tile of rows
  w0.pairs = gridDim.x / 2;
  w0.pair = blockIdx.x / 2;
  w0.nt = (vlen + kPairTile - 1) / kPairTile;
  w0.kd = (a.d + 63) / 64;

  if (warp == 0) {
    // ---- this CTA's halves of the operands --------------------------------------
    if (lane == 0) {
      const uint32_t full0 = map_to(full, 0);
      // One tile of rows: the first tile's weight does not depend on how many
      // there are, nor on the kernel before (which has started, so that what
      // precedes it on the stream has ended).
      const int early = !grad_op(OP) && a.Rp == kPairTile && w0.pair < w0.nt ? min(kStages, w0.kd) : 0;
      for (int s = 0; s < early; ++s) {
        if (rank == 0) mbar_arrive_tx(full + 8 * s, 2 * kStageBytes);   // of both CTAs
        tma_box_pair(base + s * kStageBytes + kHalfBytes, &maps.weight_k, s * 64,
                     v0 + w0.pair * kPairTile + (int)rank * 128, full0 + 8 * s);
      }
      asm volatile("griddepcontrol.wait;" ::: "memory");
      // what earlier kernels wrote with plain stores is read by the copy engine
      asm volatile("fence.proxy.async.global;" ::: "memory");
      const Work w = work_of<OP>(a, *a.n, vlen, a.d_hidden != nullptr, a.d_weight != nullptr);
      int g = 0;
      for (int i = 0; i < w.total && ok; ++i) {
        const Tile t = tile_of<OP>(a, w, i);
        const int am = t.m * kPairTile + (int)rank * 128, bn = t.n * kPairTile + (int)rank * 128;
        for (int kb = 0; kb < t.kb; ++kb, ++g) {
          const int s = g % kStages;
          if (g >= kStages && ok) ok = bar_wait<true>(empty + 8 * s, (uint32_t)((g / kStages - 1) & 1));
          if (!ok) break;
          if (rank == 0 && g >= early)
            mbar_arrive_tx(full + 8 * s, OP == kOpFewGrad && !t.dw ? 2 * kHalfBytes + (uint32_t)cols * 128 : 2 * kStageBytes);
          const uint32_t sa = base + s * kStageBytes, sb = sa + kHalfBytes, bar = full0 + 8 * s;
          const int k = (t.k0 + kb) * 64;
          if (!grad_op(OP)) {
            tma_box_pair(sa, &maps.rows_k, k, am, bar);
            if (g >= early) tma_box_pair(sb, &maps.weight_k, k, v0 + bn, bar);
          } else if (OP == kOpFewGrad && !t.dw) {
            tma_box_pair(sa, &maps.weight_n, bn, v0 + k, bar);
            tma_box_pair(sa + kHalfBytes / 2, &maps.weight_n, bn + 64, v0 + k, bar);
            tma_box_pair(sb, &maps.dz_k, k, (int)rank * (cols / 2), bar);
          } else if (!t.dw) {
            tma_box_pair(sa, &maps.dz_k, k, am, bar);
            tma_box_pair(sb, &maps.weight_n, bn, v0 + k, bar);
            tma_box_pair(sb + kHalfBytes / 2, &maps.weight_n, bn + 64, v0 + k, bar);
          } else {
            tma_box_pair(sa, &maps.dz_m, am, k, bar);
            tma_box_pair(sa + kHalfBytes / 2, &maps.dz_m, am + 64, k, bar);
            tma_box_pair(sb, &maps.rows_n, bn, k, bar);
            tma_box_pair(sb + kHalfBytes / 2, &maps.rows_n, bn + 64, k, bar);
          }
        }
      }
      // the last stages are consumed before this CTA's shared memory goes
      for (int k = (g > kStages ? g - kStages : 0); k < g; ++k)
        if (ok) ok = bar_wait<true>(empty + 8 * (k % kStages), (uint32_t)((k / kStages) & 1));
    }
  } else if (warp == 1) {
    // ---- the MMAs of both CTAs -----------------------------------------------------
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const Work w = work_of<OP>(a, *a.n, vlen, a.d_hidden != nullptr, a.d_weight != nullptr);
    if (lane == 0 && rank == 0) {
      const uint32_t empty1 = map_to(empty, 1), tfull1 = map_to(tfull, 1);
      const uint32_t empty0 = map_to(empty, 0), tfull0 = map_to(tfull, 0);
      int g = 0, c = 0;                              // stages; sums handed over
      for (int i = 0; i < w.total && ok; ++i) {
        const Tile t = tile_of<OP>(a, w, i);
        const bool few = OP == kOpFewGrad && !t.dw;
        const uint32_t idesc = !grad_op(OP) ? mma_idesc(256, 256, true, false, false)
                                            : (t.dw ? mma_idesc(256, 256, true, true, true)
                                                    : (few ? mma_idesc(256, cols, true, true, false)
                                                           : mma_idesc(256, 256, true, false, true)));
        // K = 16 further: 32 bytes along the rows, or 16 rows
        const uint64_t da = grad_op(OP) && (t.dw || few) ? 2048 >> 4 : 32 >> 4, db = grad_op(OP) && !few ? 2048 >> 4 : 32 >> 4;
        int kb = 0;
        do {                                         // (once but for the logits)
          const int end = grad_op(OP) ? t.kb : min(t.kb, kb + kSumBlocks), b = c & 1;
          if (c >= 2 && ok) ok = bar_wait<true>(tempty + 8 * b, (uint32_t)((c / 2 - 1) & 1));
          tmem_fence_after();
          const uint32_t d = tbase + (uint32_t)(b * 256);
          for (uint32_t more = 0; kb < end; ++kb, ++g) {
            const int s = g % kStages;
            if (ok) ok = bar_wait<true>(full + 8 * s, (uint32_t)((g / kStages) & 1));
            if (!ok) break;
            tmem_fence_after();
            const uint64_t ad = mma_desc(base + s * kStageBytes, kHalfBytes / 2);
            const uint64_t bd = mma_desc(base + s * kStageBytes + kHalfBytes, kHalfBytes / 2);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
              mma_pair(d, ad + ks * da, bd + ks * db, idesc, more);
              more = 1;
            }
            mma_commit_pair(empty0 + 8 * s);
            mma_commit_pair(empty1 + 8 * s);
          }
          if (!ok) break;
          mma_commit_pair(tfull0 + 8 * b);
          mma_commit_pair(tfull1 + 8 * b);
          ++c;
        } while (kb < t.kb);
      }
    }
    __syncwarp();
  } else {
    // ---- the epilogue -----------------------------------------------------------------
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int n = *a.n;
    const Work w = work_of<OP>(a, n, vlen, a.d_hidden != nullptr, a.d_weight != nullptr);
    if (!grad_op(OP)) {
      // ---- the logits' epilogue: each row's maximum and sum of a tile's entries, or P ---
      const uint32_t tempty0 = map_to(tempty, 0);
      const int q = warp & 3, group = (warp - 2) >> 2;
      const uint32_t quarter = tbase + ((uint32_t)(q * 32) << 16) + (uint32_t)(group * 64);
      float2* s_half = reinterpret_cast<float2*>(pair_smem + (base - raw) + kStages * kStageBytes);
      // this warp's rows of P on their way out: 64 bytes of each, swizzled as the boxes are
      const uint32_t obuf = base + kStages * kStageBytes + (warp - 2) * kDzBytes, orow = obuf + lane * 64;
      const uint32_t x4 = (uint32_t)(lane >> 1 & 3);
      int sums = 0;                                    // sums read
      for (int i = 0; i < w.total; ++i) {
        const Tile t = tile_of<OP>(a, w, i);
        const int row = t.m * kPairTile + (int)rank * 128 + q * 32 + lane;
        const int col = t.n * kPairTile + group * 64;
        const bool live = row < n;
        const int lab = live ? a.lab[row] - v0 : -1;   // (the loss: v0 is 0)
        float z[64];
        for (int kb = 0; kb < t.kb; kb += kSumBlocks, ++sums) {
          const int b = sums & 1;
          if (ok) ok = bar_wait<true>(tfull + 8 * b, (uint32_t)((sums / 2) & 1));
          ok = __all_sync(kFull, ok);
          if (!ok) break;
          tmem_fence_after();
          const uint32_t src = quarter + b * 256;
          if (kb == 0) {                             // (a loop of its own: with one for both the sums spilled)
            float y[32];
#pragma unroll
            for (int c = 0; c < 64; c += 32) {
              tmem_ld32(src + c, y);
#pragma unroll
              for (int k = 0; k < 32; ++k) z[c + k] = y[k];
            }
          } else {
#pragma unroll
            for (int c = 0; c < 64; c += 16) {
              float y[16];
              tmem_ld16_ahead(src + c, y);
              tmem_ld_wait(y);
#pragma unroll
              for (int k = 0; k < 16; ++k) z[c + k] += y[k];
            }
          }
          tmem_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(tempty0 + 8 * b);   // this warp's columns have been read
        }
        if (OP == kOpDz) {
          if (!ok) break;
          const float lse = live ? a.plse[row] : 0.f, gr = live ? a.pgrad[row] : 0.f;
#pragma unroll
          for (int c = 0; c < 64; c += 32) {
#pragma unroll
            for (int k = c; k < c + 32; ++k)
              z[k] = live && col + k < vlen ? (ex2((z[k] - lse) * kLog2e) - (lab == col + k ? 1.f : 0.f)) * gr : 0.f;
            if (lane == 0) tma_store_wait_read();
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float* v = z + c + 8 * k;
              st_shared(orow + (((uint32_t)k ^ x4) << 4), pack_bf(v[0], v[1]), pack_bf(v[2], v[3]),
                        pack_bf(v[4], v[5]), pack_bf(v[6], v[7]));
            }
            smem_to_copies();
            __syncwarp();
            if (lane == 0) {
              tma_store(&maps.dz_out, col + c, row - lane, obuf);
              tma_store_commit();
            }
          }
          continue;
        }
        // (after a wait that gave up: on to the barrier, where another warp waits, and nothing is written)
        if (ok && lab >= col && lab < col + 64) {
          float zl = z[0];
#pragma unroll
          for (int k = 1; k < 64; ++k) zl = lab == col + k ? z[k] : zl;
          a.zlab[row] = zl;
        }
        if (col + 64 > vlen) {
#pragma unroll
          for (int k = 0; k < 64; ++k)
            if (col + k >= vlen) z[k] = -pos_inf();
        }
        float m4[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
        for (int k = 4; k < 64; ++k) m4[k & 3] = fmaxf(m4[k & 3], z[k]);
        float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * kLog2e;
        const float ref = mx > -pos_inf() ? mx : 0.f;
        float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 64; ++k) s4[k & 3] += ex2(fmaf(z[k], kLog2e, -ref));
        float sum = (s4[0] + s4[1]) + (s4[2] + s4[3]);
        // the second 64 of 128 columns join the first (two buffers in turn: one barrier a tile)
        float2* mine = s_half + ((i & 1) * 2 + (group >> 1)) * 128 + q * 32 + lane;
        if (group & 1) *mine = make_float2(mx, sum);
        asm volatile("bar.sync %0, 64;" ::"r"(1 + (group >> 1) * 4 + q) : "memory");
        if (ok && !(group & 1) && live && col < vlen) {
          const float2 x = *mine;
          fold(mx, sum, x.x, x.y);
          a.part[(size_t)(col / kHeadPart) * a.Rp + row] = make_float2(mx, sum);
        }
      }
      if (OP == kOpDz && lane == 0) tma_store_wait();
    } else {
      const uint32_t tempty0 = map_to(tempty, 0);
      const int q = warp & 3, half = (warp - 2) >> 2;
      // this warp's rows on their way out: 128 bytes of each, swizzled as the boxes are
      const uint32_t obuf = base + kStages * kStageBytes + (warp - 2) * kOutBytes, orow = obuf + lane * 128;
      const uint32_t x8 = (uint32_t)(lane & 7);
      // 32 columns of 32 rows as bf16; a box of 64 goes out with every second call
      auto out_bf16 = [&](const float (&v)[32], int c, int y, int x, bool inside, const CUtensorMap* map) {
        if ((c & 32) == 0) {
          if (lane == 0) tma_store_wait_read();
          __syncwarp();
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
          st_shared(orow + (((uint32_t)(k + (c & 32) / 8) ^ x8) << 4), pack_bf(v[8 * k], v[8 * k + 1]),
                    pack_bf(v[8 * k + 2], v[8 * k + 3]), pack_bf(v[8 * k + 4], v[8 * k + 5]),
                    pack_bf(v[8 * k + 6], v[8 * k + 7]));
        if (c & 32) {
          smem_to_copies();
          __syncwarp();
          if (lane == 0 && inside) {                   // (part of a box may lie outside, not all of it)
            tma_store(map, x - 32, y, obuf);
            tma_store_commit();
          }
        }
      };
      for (int i = 0; i < w.total; ++i) {
        const Tile t = tile_of<OP>(a, w, i);
        const int b = i & 1;
        if (ok) ok = bar_wait<true>(tfull + 8 * b, (uint32_t)((i / 2) & 1));
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        tmem_fence_after();
        const int row0 = t.m * kPairTile + (int)rank * 128 + q * 32;
        const int col = t.n * kPairTile + half * 128;
        const uint32_t src = tbase + ((uint32_t)(q * 32) << 16) + (uint32_t)(b * 256 + half * 128);
        // few rows, d_hidden: a lane is an entry of d, the columns are rows, every second group of 32 for each half
        const bool few = OP == kOpFewGrad && !t.dw;
        if (few) {
          const int x = t.n * kPairTile + (int)rank * 128 + q * 32 + lane;
          const uint32_t at = tbase + ((uint32_t)(q * 32) << 16) + (uint32_t)(b * 256);
#pragma unroll 1
          for (int c = 32 * half; c < cols; c += 64) {
            float z[32];
            tmem_ld32(at + c, z);
            float* dst = a.dh + ((size_t)t.part * a.Rp + c) * a.d + x;
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (x < a.d && c + k < a.R) {
                const float y = t.kb > 0 ? z[k] : 0.f;
                dst[(size_t)k * a.d] = first ? y : dst[(size_t)k * a.d] + y;
              }
          }
          tmem_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(tempty0 + 8 * b);
          continue;
        }
#pragma unroll 1
        for (int c = 0; c < 128; c += 32) {
          float z[32];
          if (t.kb > 0) {
            tmem_ld32(src + c, z);
          } else {
#pragma unroll
            for (int k = 0; k < 32; ++k) z[k] = 0.f;
          }
          if (c == 96) {
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(tempty0 + 8 * b);   // this warp's columns have been read
          }
          const int j0 = col + c;
          if (t.dw) {
            out_bf16(z, c, v0 + row0, j0, v0 + row0 < a.V && (j0 & ~63) < a.d, &maps.dw_out);
          } else {
            if (lane == 0) tma_store_wait_read();
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 8; ++k)
              st_shared(orow + (((uint32_t)k ^ x8) << 4), __float_as_uint(z[4 * k]), __float_as_uint(z[4 * k + 1]),
                        __float_as_uint(z[4 * k + 2]), __float_as_uint(z[4 * k + 3]));
            smem_to_copies();
            __syncwarp();
            if (lane == 0 && j0 < a.d) {
              if (first)
                tma_store(&maps.dh_out, j0, t.part * a.Rp + row0, obuf);
              else                                     // (one addition a piece: the order is that of the pieces)
                tma_add(&maps.dh_out, j0, t.part * a.Rp + row0, obuf);
              tma_store_commit();
            }
          }
        }
      }
      if (lane == 0) tma_store_wait();
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
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tbase), "r"(kTmemCols) : "memory");
}

// ---- few rows ------------------------------------------------------------------------
//
// With up to 128 rows the products are bound by memory as long as the tensor
// cores do no more than they must: a tile of 256 rows takes 512 cycles for 64 of
// K however few of them are live, in which memory delivers half a tile more.  So the roles change: the MMA's M is the
// vocabulary (or d, for d_hidden) and its N the rows, in multiples of 32.
//   logits    A = weight (128 entries a CTA at most), B = packed rows, K = d
//   d_hidden  A = weight (its rows run along M = d), B = P, K = entries, together
//             with d_weight's tiles in head_pair_kernel
// (d_weight's product has few rows as its K, and stays as it is.)  The warps and
// barriers are those of head_pair_kernel.  A thread of the epilogue holds one
// entry's logits of all rows; a row's maximum and sum go across the warp's lanes
// by halving the rows in play with each exchange, 31 exchanges for 32 rows, which
// leaves row c with lane c.  All of a pair's tiles are folded before anything is
// written.
// (us, and by tiles of 256 rows: R=16 d=512 V=8000 loss 10.5, 12.7, gradients 20.6,
// 26.8; R=128 12.5, 14.3 and 25, 27; R=16 d=2048 V=128256 85, 102 and 267, 467; R=128
// 87, 106 and 285, 365.)
// The rows are not packed: an ignored row is a column of the MMA that is not
// read, and a row of zeros in P.  d_weight's product, whose K the rows are, takes
// a copy of them in which the ignored ones are zeros.
enum FewOp { kFewStats, kFewDz };
constexpr int kFewRows = 128;
constexpr int kFewStages = 9;
constexpr int kFewBBytes = kFewRows / 2 * 128;         // this CTA's half of the rows
constexpr int kFewStage = kHalfBytes + kFewBBytes;
constexpr size_t kFewTable = (size_t)kFewRows * 16;    // each row's label, lse and gradient
constexpr size_t kFewRed = (size_t)kEpiWarps * 2 * 32 * 8;
constexpr size_t kFewSmem =
    1024 + (size_t)kFewStages * kFewStage + kFewTable + kFewRed + 8 * (2 * kFewStages + 4) + 16;
static_assert(kFewSmem <= 227 * 1024, "shared memory");

// w[c] of every lane reduced over the warp's lanes: lane c gets row c's
template <typename F>
__device__ __forceinline__ float across(float (&w)[32], int lane, F f) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float keep = up ? w[i + o] : w[i], send = up ? w[i] : w[i + o];
      w[i] = f(keep, __shfl_xor_sync(kFull, send, o));
    }
  }
  return w[0];
}

struct FewPlan {
  int height;            // entries of the vocabulary per CTA and tile
  int cols;              // rows, a multiple of 32
  int tiles;
};
template <int OP>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
    head_few_kernel(const HeadLossArgs a, const FewPlan p, const int v0, const int vlen, const int first,
                    const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b) {
  extern __shared__ __align__(1024) unsigned char few_smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster_rank(), pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  const uint32_t raw = smem_addr(few_smem);
  const uint32_t base = (raw + 1023u) & ~1023u;
  unsigned char* sm = few_smem + (base - raw);
  int4* s_table = reinterpret_cast<int4*>(sm + kFewStages * kFewStage);
  float2* s_red = reinterpret_cast<float2*>(sm + kFewStages * kFewStage + kFewTable);
  const uint32_t bars = base + (uint32_t)(kFewStages * kFewStage + kFewTable + kFewRed);
  const uint32_t full = bars, empty = bars + 8 * kFewStages, tfull = bars + 16 * kFewStages, tempty = tfull + 16;
  uint32_t* s_taddr = reinterpret_cast<uint32_t*>(sm + (bars - base) + 8 * (2 * kFewStages + 4));
  if (tid == 0) {
    for (int k = 0; k < kFewStages; ++k) {
      mbar_init(full + 8 * k, 1);
      mbar_init(empty + 8 * k, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(tfull + 8 * b, 1);
      mbar_init(tempty + 8 * b, 2 * kEpiWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(s_taddr)),
                 "r"(256)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tmem_fence_before();
  cluster_sync_all();
  tmem_fence_after();
  const uint32_t tbase = *s_taddr;                  // two accumulators of 128 columns
  const int mine = p.tiles > pair ? (p.tiles - pair + pairs - 1) / pairs : 0;
  const int kb = (a.d + 63) / 64;                   // blocks of K
  bool ok = true;

  if (warp == 0) {
    if (lane == 0) {
      const uint32_t full0 = map_to(full, 0);
      const uint32_t bytes = (uint32_t)(p.height * 256 + p.cols * 128);    // of both CTAs
      auto load_a = [&](int t, int k, int s) {
        if (rank == 0) mbar_arrive_tx(full + 8 * s, bytes);
        tma_box_pair(base + s * kFewStage, &map_a, k * 64, v0 + (t * 2 + rank) * p.height, full0 + 8 * s);
      };
      // the weight's first stages do not wait for the kernel before (which has
      // started, so that what precedes it on the stream has ended)
      const int early = mine > 0 ? min(kFewStages, kb) : 0;
      for (int s = 0; s < early; ++s) load_a(pair, s, s);
      asm volatile("griddepcontrol.wait;" ::: "memory");
      asm volatile("fence.proxy.async.global;" ::: "memory");
      int g = 0;
      for (int i = 0; i < mine && ok; ++i) {
        for (int k = 0; k < kb; ++k, ++g) {
          const int s = g % kFewStages;
          if (g >= kFewStages && ok) ok = bar_wait<true>(empty + 8 * s, (uint32_t)((g / kFewStages - 1) & 1));
          if (!ok) break;
          if (g >= early) load_a(pair + i * pairs, k, s);
          tma_box_pair(base + s * kFewStage + kHalfBytes, &map_b, k * 64, rank * (p.cols / 2), full0 + 8 * s);
        }
      }
      for (int k = (g > kFewStages ? g - kFewStages : 0); k < g; ++k)
        if (ok) ok = bar_wait<true>(empty + 8 * (k % kFewStages), (uint32_t)((k / kFewStages) & 1));
    }
  } else if (warp == 1) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (rank == 0) {
      const bool leader = elect_lane();
      const uint32_t empty1 = map_to(empty, 1), tfull1 = map_to(tfull, 1);
      const uint32_t empty0 = map_to(empty, 0), tfull0 = map_to(tfull, 0);
      const uint32_t idesc = mma_idesc(256, p.cols, true, false, false);
      int s = 0;
      uint32_t phase = 0;
      const int parts = (kb + kSumBlocks - 1) / kSumBlocks;
      for (int c = 0, k1 = 0; c < mine * parts; ++c) {       // sums
        const int b = c & 1, k0 = k1 == kb ? 0 : k1;
        if (c >= 2 && ok) ok = bar_wait<true>(tempty + 8 * b, (uint32_t)((c / 2 - 1) & 1));
        tmem_fence_after();
        const uint32_t d = tbase + (uint32_t)(b * 128);
        k1 = min(kb, k0 + kSumBlocks);
        for (int k = k0; k < k1; ++k) {
          if (ok) ok = bar_wait<true>(full + 8 * s, phase);
          tmem_fence_after();
          const uint64_t ad = mma_desc(base + s * kFewStage, 0);
          const uint64_t bd = mma_desc(base + s * kFewStage + kHalfBytes, 0);
          if (leader && ok) {
#pragma unroll
            for (int j = 0; j < 4; ++j) mma_pair(d, ad + (uint64_t)(2 * j), bd + (uint64_t)(2 * j), idesc, k > k0 || j > 0);
            mma_commit_pair(empty0 + 8 * s);
            mma_commit_pair(empty1 + 8 * s);
          }
          __syncwarp();
          if (++s == kFewStages) {
            s = 0;
            phase ^= 1;
          }
        }
        if (leader && ok) {
          mma_commit_pair(tfull0 + 8 * b);
          mma_commit_pair(tfull1 + 8 * b);
        }
        __syncwarp();
      }
    }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2, e = tid - 64;
    const uint32_t tempty0 = map_to(tempty, 0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int c = e; c < p.cols; c += 32 * kEpiWarps) {
      int4 x = make_int4(-1, 0, 0, 0);
      const int label = c < a.R ? a.labels[c] : a.ignore;
      if (kept(a, label)) {
        x.x = label - v0;
        x.w = 1;
        if (OP == kFewDz) {
          x.y = __float_as_int(a.lse_in[c]);
          x.z = __float_as_int(a.grad[c]);
        }
      } else if (label != a.ignore && blockIdx.x == 0) {
        report(a.err, 1u);
      }
      s_table[c] = x;
    }
    if (OP == kFewDz && a.d_weight && first) {     // a CTA a row, and some of zeros
      for (int r = blockIdx.x; r < (a.R + 63) / 64 * 64; r += gridDim.x) {
        const bool keep = r < a.R && kept(a, a.labels[r]);
        const uint4* src = reinterpret_cast<const uint4*>(a.hidden + (size_t)(keep ? r : 0) * a.d);
        for (int j = e; j < a.d / 8; j += 32 * kEpiWarps)
          reinterpret_cast<uint4*>(a.packed + (size_t)r * a.d)[j] = keep ? src[j] : make_uint4(0, 0, 0, 0);
      }
    }
    if (OP == kFewDz && first && blockIdx.x == 0 && e == 0) *a.n = a.R;
    asm volatile("bar.sync 1, 256;" ::: "memory");
    // this warp's rows: every second group of 32
    float mx[2] = {-pos_inf(), -pos_inf()}, sum[2] = {0.f, 0.f};
    for (int i = 0, sums = 0; i < mine; ++i) {
      const int t = pair + i * pairs;
      const int at = q * 32 + lane;                  // this thread's entry within the CTA's part
      const int v = (t * 2 + rank) * p.height + at;
      const bool live = at < p.height && v < vlen;
      float acc[2][32];                              // the logits, part by part
      for (int k0 = 0; k0 < kb; k0 += kSumBlocks, ++sums) {
        const int b = sums & 1;
        if (ok) ok = bar_wait<true>(tfull + 8 * b, (uint32_t)((sums / 2) & 1));
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        tmem_fence_after();
        const uint32_t src = tbase + ((uint32_t)(q * 32) << 16) + (uint32_t)(b * 128);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int c0 = 32 * (2 * u + half);
          if (c0 < p.cols) {
            float y[32];
            tmem_ld32(src + c0, y);
#pragma unroll
            for (int k = 0; k < 32; ++k) acc[u][k] = k0 == 0 ? y[k] : acc[u][k] + y[k];
          }
        }
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(tempty0 + 8 * b);       // this warp's columns have been read
      }
      if (!ok) break;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int c0 = 32 * (2 * u + half);
        if (c0 >= p.cols) break;
        float (&z)[32] = acc[u];
        if (OP == kFewStats) {
          const int lab = s_table[c0 + lane].x, from = v - lane;
          unsigned hit = __ballot_sync(kFull, lab >= from && lab < from + 32 && q * 32 + lab - from < p.height);
          while (hit) {                              // a row whose label is an entry of this warp's
            const int c = __ffs(hit) - 1;
            hit &= hit - 1;
            float zc = z[0];
#pragma unroll
            for (int k = 1; k < 32; ++k) zc = c == k ? z[k] : zc;
            if (__shfl_sync(kFull, lab, c) == v) a.zlab[c0 + c] = zc;
          }
          float x[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            z[k] = live ? z[k] : -pos_inf();
            x[k] = z[k] * kLog2e;
          }
          const float tm = across(x, lane, [](float f, float g) { return fmaxf(f, g); });
          const float nm = fmaxf(mx[u], tm), ref = nm > -pos_inf() ? nm : 0.f;
#pragma unroll
          for (int k = 0; k < 32; ++k) x[k] = ex2(fmaf(z[k], kLog2e, -__shfl_sync(kFull, ref, k)));
          const float ts = across(x, lane, [](float f, float g) { return f + g; });
          sum[u] = (sum[u] != 0.f ? sum[u] * ex2(mx[u] - ref) : 0.f) + ts;
          mx[u] = nm;
        } else {
          uint16_t* dst = a.dz + (size_t)c0 * a.Vc + v;
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            const int4 x = s_table[c0 + k];
            const float pr = (ex2((z[k] - __int_as_float(x.y)) * kLog2e) - (x.x == v ? 1.f : 0.f)) * __int_as_float(x.z);
            if (live) dst[(size_t)k * a.Vc] = x.w ? (uint16_t)pack_bf(pr, 0.f) : (uint16_t)0;
          }
        }
      }
    }
    if (OP == kFewStats) {
#pragma unroll
      for (int u = 0; u < 2; ++u) s_red[((warp - 2) * 2 + u) * 32 + lane] = make_float2(mx[u], sum[u]);
      asm volatile("bar.sync 1, 256;" ::: "memory");
      // row e: the four warps of its group, quarter by quarter (warps 2..5 or 6..9)
      if (e < p.cols) {
        const int g = e >> 5, w = (g & 1) * 4, u = g >> 1;
        float m = -pos_inf(), s = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 x = s_red[((w + k) * 2 + u) * 32 + (e & 31)];
          fold(m, s, x.x, x.y);
        }
        a.part[(size_t)blockIdx.x * a.Rp + e] = make_float2(m, s);
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
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tbase), "r"(256) : "memory");
}

// ---- a row's tiles merged -----------------------------------------------------------
// Four rows a CTA (32 bytes of each tile's statistics), 64 tiles at a time.
// The loss is a difference of two numbers that a trained head makes nearly equal:
// it is formed from the maximum and the label's logit first.
// kFew: the rows are not packed
constexpr int kMergeThreads = 256;
template <bool kFew>
__global__ void __launch_bounds__(kMergeThreads) head_merge_kernel(const HeadLossArgs a, int parts) {
  __shared__ float s_m[kMergeThreads / 32][4], s_s[kMergeThreads / 32][4];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x * 4 + (tid & 3);
  const bool keep = r < a.R && kept(a, a.labels[r]);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int p = keep ? (kFew ? r : a.pos[r]) : -1;
  const float zl = tid < 4 && keep ? a.zlab[p] : 0.f;          // (requested with the statistics)
  float m = -pos_inf(), s = 0.f;
  if (keep) {
    constexpr int kBatch = 8;
    for (int t0 = tid >> 2; t0 < parts; t0 += kBatch * (kMergeThreads / 4)) {
      float2 x[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int t = t0 + j * (kMergeThreads / 4);
        x[j] = t < parts ? __ldcg(a.part + (size_t)t * a.Rp + p) : make_float2(-pos_inf(), 0.f);
      }
      float mm = m;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) mm = fmaxf(mm, x[j].x);
      s = s != 0.f ? s * ex2(m - mm) : 0.f;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) s += x[j].y != 0.f ? x[j].y * ex2(x[j].x - mm) : 0.f;
      m = mm;
    }
  }
#pragma unroll
  for (int o = 16; o >= 4; o >>= 1) fold(m, s, __shfl_xor_sync(kFull, m, o), __shfl_xor_sync(kFull, s, o));
  if (lane < 4) {
    s_m[warp][lane] = m;
    s_s[warp][lane] = s;
  }
  __syncthreads();
  if (tid < 4 && r < a.R) {
    float lse = 0.f, loss = 0.f;
    if (keep) {
#pragma unroll
      for (int w = 1; w < kMergeThreads / 32; ++w) fold(m, s, s_m[w][tid], s_s[w][tid]);
      const float l = logf(s);
      lse = m * kLn2 + l;
      loss = fmaf(fmaf(-zl, kLog2e, m), kLn2, l);
    }
    a.lse[r] = lse;
    if (a.loss) a.loss[r] = loss;
  }
}

// ---- the hidden states' gradient, rounded and put back in place -------------------
// kLanes threads share four columns' parts (four where there are many parts: their
// loads are in flight together).
constexpr int kUnpackThreads = 128;
template <bool kFew, int kLanes>
__global__ void __launch_bounds__(kUnpackThreads) head_unpack_kernel(const HeadLossArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, sub = kLanes == 1 ? 0 : lane >> 3;
  constexpr int kCols = 32 / kLanes;                 // groups of four columns a warp
  const int j = (int)((blockIdx.x * (kUnpackThreads / 32) + (threadIdx.x >> 5)) * kCols + (lane & (kCols - 1))) * 4;
  const size_t step = (size_t)a.Rp * a.d;
  for (int r = blockIdx.y; r < a.R; r += gridDim.y) {
    const int p = kFew ? (kept(a, a.labels[r]) ? r : -1) : a.pos[r];
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (p >= 0 && j < a.d) {
      const float* src = a.dh + (size_t)p * a.d + j;
#pragma unroll 4
      for (int k = sub; k < a.split; k += kLanes) {
        const float4 y = __ldcg(reinterpret_cast<const float4*>(src + k * step));
        x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
      }
    }
    if (kLanes > 1) {
#pragma unroll
      for (int o = 8; o <= 16; o <<= 1) {
        x.x += __shfl_xor_sync(kFull, x.x, o);
        x.y += __shfl_xor_sync(kFull, x.y, o);
        x.z += __shfl_xor_sync(kFull, x.z, o);
        x.w += __shfl_xor_sync(kFull, x.w, o);
      }
    }
    if (sub == 0 && j < a.d)
      *reinterpret_cast<uint2*>(a.d_hidden + (size_t)r * a.d + j) = make_uint2(pack_bf(x.x, x.y), pack_bf(x.z, x.w));
  }
}

unsigned tiles(int64_t n, int t) { return (unsigned)((n + t - 1) / t); }
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
cudaError_t launch_pack(const HeadLossArgs& a, cudaStream_t s) {
  int rows = kPackWarps;
  while ((int64_t)rows * 1024 < a.R) rows *= 2;
  const int ctas = (int)tiles(a.R, rows);
  head_pack_kernel<<<ctas + kPackZero, kPackThreads, 0, s>>>(a, rows, ctas);
  return cudaGetLastError();
}

template <bool kFew>
cudaError_t launch_unpack(const HeadLossArgs& a, cudaStream_t s) {
  const bool shared = a.split >= 4;
  const dim3 grid(tiles(a.d, kUnpackThreads * (shared ? 1 : 4)), (unsigned)(a.R < 65535 ? a.R : 65535));
  return shared ? launch(true, head_unpack_kernel<kFew, 4>, grid, kUnpackThreads, 0, s, a)
                : launch(true, head_unpack_kernel<kFew, 1>, grid, kUnpackThreads, 0, s, a);
}

bool encode_maps(const HeadLossArgs& a, bool backward, Maps* m) {
  const CUtensorMapDataType t = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  bool ok = tma_matrix(&m->rows_k, t, 2, a.packed, a.d, a.Rp, 128) && tma_matrix(&m->weight_k, t, 2, a.weight, a.d, a.V, 128);
  if (!backward) {
    m->rows_n = m->weight_n = m->dz_k = m->dz_m = m->dz_out = m->dw_out = m->dh_out = m->rows_k;   // not read
    return ok;
  }
  m->dw_out = m->dh_out = m->rows_k;
  if (a.d_weight) ok = ok && tma_matrix(&m->dw_out, t, 2, a.d_weight, a.d, a.V, 32);
  if (a.d_hidden)
    ok = ok && tma_matrix(&m->dh_out, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, a.dh, a.d, (int64_t)a.split * a.Rp, 32);
  return ok && tma_matrix(&m->rows_n, t, 2, a.packed, a.d, a.Rp, 64) && tma_matrix(&m->weight_n, t, 2, a.weight, a.d, a.V, 64) &&
         tma_matrix(&m->dz_k, t, 2, a.dz, a.Vc, a.Rp, 128) && tma_matrix(&m->dz_m, t, 2, a.dz, a.Vc, a.Rp, 64) &&
         tma_matrix(&m->dz_out, t, 2, a.dz, a.Vc, a.Rp, 32, 0, 64);
}

// `most`: tiles at most; one pair of CTAs for each two SMs runs through them
template <typename K>
cudaError_t allow_smem(K kernel, size_t smem, unsigned long long* done, int* pairs) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = 1ull << (dev & 63);
  if (!(__atomic_load_n(done, __ATOMIC_ACQUIRE) & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    __atomic_fetch_or(done, bit, __ATOMIC_ACQ_REL);
  }
  *pairs = sms / 2 > 0 ? sms / 2 : 1;
  return cudaSuccess;
}
template <int OP>
cudaError_t launch_pairs(const HeadLossArgs& a, int v0, int vlen, int first, int cols, int64_t most, const Maps& maps,
                         cudaStream_t s) {
  static unsigned long long done = 0ull;
  int pairs = 0;
  const cudaError_t e = allow_smem(head_pair_kernel<OP>, kPairSmem, &done, &pairs);
  if (e != cudaSuccess) return e;
  if (pairs > most) pairs = (int)most;
  return launch(true, head_pair_kernel<OP>, (unsigned)(2 * pairs), 64 + 32 * epi_warps(OP), kPairSmem, s, a, v0, vlen, first, cols, maps);
}

// *ctas gets the CTAs, each of which leaves one partial statistic a row
// (kFewParts at most)
template <int OP>
cudaError_t launch_few(bool early, const HeadLossArgs& a, int v0, int vlen, int first, int* ctas, cudaStream_t s) {
  static unsigned long long done = 0ull;
  int pairs = 0;
  const cudaError_t e = allow_smem(head_few_kernel<OP>, kFewSmem, &done, &pairs);
  if (e != cudaSuccess) return e;
  if (pairs > kFewParts / 2) pairs = kFewParts / 2;
  FewPlan p;
  p.cols = (a.R + 31) / 32 * 32;
  // the vocabulary spread evenly over the pairs' rounds
  const int64_t wave = (int64_t)pairs * 256, waves = (vlen + wave - 1) / wave;
  p.height = (int)(((vlen + 2 * pairs * waves - 1) / (2 * pairs * waves) + 7) / 8 * 8);
  p.tiles = (int)tiles(vlen, 2 * p.height);
  const CUtensorMapDataType t = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  CUtensorMap ma, mb;
  if (!tma_matrix(&ma, t, 2, a.weight, a.d, a.V, p.height) || !tma_matrix(&mb, t, 2, a.hidden, a.d, a.R, p.cols / 2))
    return cudaErrorInvalidValue;
  if (pairs > p.tiles) pairs = p.tiles;
  if (ctas) *ctas = 2 * pairs;
  return launch(early, head_few_kernel<OP>, (unsigned)(2 * pairs), kPairThreads, kFewSmem, s, a, p, v0, vlen, first, ma, mb);
}
}  // namespace

// Parts that d_hidden's sum over a piece is cut into, so that its tiles fill the
// pairs of SMs: the least of rounds / parts, each part charged for its sums' way
// through memory (8 bytes a sum and piece at 5 TB/s, against 2 Vc operations at
// 1.7 PFLOP/s).  R=4096 d=2048 V=128256, both gradients: one part 2.96 ms, four
// 3.07.  A part has at least four blocks of 64.  The 76 pairs are GB300's 152 SMs and
// not asked of the device: the parts decide the workspace's size, which depends on the
// call's sizes alone.  (The launch counts the device's SMs; with fewer of them the
// parts are a worse choice, and right.)
int head_split(int Rp, int d, int Vc) {
  const int64_t t = (int64_t)(Rp / kPairTile) * ((d + kPairTile - 1) / kPairTile);
  const int most = Vc / 256 < 32 ? Vc / 256 : 32;
  int best = 1;
  double least = 0.0;
  for (int k = 1; k <= most; ++k) {
    const double cost = (double)((t * k + 75) / 76) / k * (1.0 + 1400.0 / Vc * k);
    if (k == 1 || cost < least) {
      best = k;
      least = cost;
    }
  }
  return best;
}

// one wait at a barrier that has its one arrival, or never gets it
__global__ void test_wait_kernel(unsigned* err, int arrive, long long limit) {
  __shared__ __align__(8) unsigned long long s_bar;
  const uint32_t bar = smem_addr(&s_bar);
  if (threadIdx.x == 0) {
    mbar_init(bar, 1);
    if (arrive) mbar_arrive_local(bar);
  }
  __syncwarp();
  if (!bar_wait<false>(bar, 0, limit)) {
    report(err, 4u);
    let_settle();
  }
}
cudaError_t launch_test_wait(unsigned* err, int arrive, cudaStream_t s) {
  test_wait_kernel<<<1, 32, 0, s>>>(err, arrive, 1ll << 24);
  return cudaGetLastError();
}

cudaError_t take_head_loss_errors(unsigned* flags, cudaStream_t s) { return take_errors(flags, s); }

cudaError_t launch_head_loss(const HeadLossArgs& a, cudaStream_t s) {
  if (a.R <= kFewRows) {
    int parts = 0;
    const cudaError_t e = launch_few<kFewStats>(false, a, 0, a.V, 1, &parts, s);
    if (e != cudaSuccess) return e;
    return launch(true, head_merge_kernel<true>, tiles(a.R, 4), kMergeThreads, 0, s, a, parts);
  }
  Maps maps;
  if (!encode_maps(a, false, &maps)) return cudaErrorInvalidValue;
  cudaError_t e = launch_pack(a, s);
  if (e != cudaSuccess) return e;
  e = launch_pairs<kOpStats>(a, 0, a.V, 1, 0, (int64_t)(a.Rp / kPairTile) * tiles(a.V, kPairTile), maps, s);
  if (e != cudaSuccess) return e;
  return launch(true, head_merge_kernel<false>, tiles(a.R, 4), kMergeThreads, 0, s, a, (int)tiles(a.V, kHeadPart));
}

cudaError_t launch_head_loss_backward(const HeadLossArgs& a, cudaStream_t s) {
  const bool few = a.R <= kFewRows;
  const int cols = (a.R + 31) / 32 * 32;
  Maps maps;
  if (!encode_maps(a, true, &maps)) return cudaErrorInvalidValue;
  cudaError_t e = few ? cudaSuccess : launch_pack(a, s);
  if (e != cudaSuccess) return e;
  const int64_t mt = few ? 1 : a.Rp / kPairTile, dt = tiles(a.d, kPairTile);
  for (int64_t v0 = 0; v0 < a.V; v0 += a.Vc) {
    const int vlen = (int)min((int64_t)a.Vc, a.V - v0), first = v0 == 0;
    const int64_t vt = tiles(vlen, kPairTile);
    const int64_t most = (a.d_hidden ? mt * dt * a.split : 0) + (a.d_weight ? vt * dt : 0);
    if (few) {
      // P's entries and rows that are not written read as zeros
      const CUtensorMapDataType t = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
      if (!tma_matrix(&maps.dz_k, t, 2, a.dz, vlen, cols, cols / 2, a.Vc) ||
          !tma_matrix(&maps.dz_m, t, 2, a.dz, vlen, cols, 64, a.Vc))
        return cudaErrorInvalidValue;
      e = launch_few<kFewDz>(!first, a, (int)v0, vlen, first, nullptr, s);
      if (e == cudaSuccess) e = launch_pairs<kOpFewGrad>(a, (int)v0, vlen, first, cols, most, maps, s);
    } else {
      e = launch_pairs<kOpDz>(a, (int)v0, vlen, first, 0, mt * vt, maps, s);
      if (e == cudaSuccess) e = launch_pairs<kOpGrad>(a, (int)v0, vlen, first, 0, most, maps, s);
    }
    if (e != cudaSuccess) return e;
  }
  if (!a.d_hidden) return cudaSuccess;
  return few ? launch_unpack<true>(a, s) : launch_unpack<false>(a, s);
}

}  // namespace cmsd
