// linear_loss.cu -- cross entropy of a head's logits from the hidden rows and the
// head's weight, with the gradients of both.  The loss alone keeps no logits; the
// gradients keep their exponentials in bf16, in the workspace.
//
//   z = h W^T,  L_t = log sum_v exp z_tv - z_ty,  loss = sum_t w_t L_t
//   dz_tv = w_t (softmax(z_t)_v - [v = y]),  dh = dz W,  dW = dz^T h
//
// Three matrix products of 2 T V H operations each, on the tensor cores.  A pass
// over the logits for their sums and a second one for dz would make it four; this
// needs one, because dz is a row factor times numbers that are known before the
// sum: with the label's logit z_y as the row's reference (T dot products, first),
//   e_tv = exp(z_tv - z_ty),  S_t = sum over v != y of e_tv,  L_t = log(1 + S_t)
//   dz_tv = w_t / (1 + S_t) * (v = y ? -S_t : e_tv)
// The first product's epilogue leaves e in bf16 and the sums of its columns; the
// sums' kernel puts -S at the label and scales a copy of h by w / (1 + S).  Then
//   dh = w / (1 + S) * (e W)   (the factor after the product)
//   dW = e^T (w / (1 + S) h)
// The label stays out of S, so that a nearly sure row's loss and gradient keep
// their digits.  Two values are rounded to bf16 on the way, as the tensor cores
// take them: e and, for dW, the scaled rows.
//
// z_y lies below log sum exp z, so e can grow: up to e^L.  Rows with L above
// kMostLoss (a label of probability 1e-26) take the row's largest logit as the
// reference instead, in a second run of the first product over their tiles.
//
// Rows without a label take part in nothing: the others are moved together first.
// The matrix e, [rows, vocab] bf16, has at most kMostCells elements: more rows are
// taken in chunks, and dW is then summed in fp32.
//
// The products (one kernel): a pair of CTAs per 256 x 256 tile, persistent; one warp
// issues TMA copies of 64-deep slices into a ring of kStages, one the pair's MMAs
// (M = N = 256, cta_group::2), eight read the accumulators, which are double
// buffered in tensor memory.  Operands lie as they are, along the contraction (K-major)
// or across it (MN-major): no transposed copies.
#include <cudaTypedefs.h>

#include <atomic>
#include <cfloat>

#include "train.cuh"

namespace slimwise {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMostLoss = 60.0f;
// The tensor cores' fp32 sums are cut, not rounded, at each step of the contraction that
// adds something: a logit of a dense row is too small in magnitude by 1.03e-9 of itself
// for each element of the width where it grows steadily, 0.9e-9 where it wanders (widths of
// 512 to 4096 alike), while the label's, of plain sums, is not.  The expected loss is given
// back, by the pieces of 8 elements of the row that are not all zeros.  It holds beyond: mean
// error of 300 row losses (10 to 16) at 8192 3e-7 in place of -1.1e-5, of 200 at 16384
// under 1e-7 in place of -2.1e-5.  It is an expectation: a sum that happens to be exact gets
// its share all the same, 1e-9 of the logit for each element.
constexpr float kTruncated = 1.0e-9f;
__host__ __device__ inline float given_back(int elements) { return fmaf((float)elements, kTruncated, 1.0f); }
constexpr int64_t kMostCells = 1ll << 30;
constexpr int kTile = 256;       // rows and columns of a pair's tile
constexpr int kHalf = 128;       // of a CTA's share of an operand
constexpr int kDepth = 64;       // slice of the contraction: 128 bytes
constexpr int kStages = 6;
// Roles swapped: the vocabulary (for dh: the width) is M, which fills the tensor cores'
// rows and the accumulators' lanes, and tiles of `rows_tile` rows, a multiple of 32, are
// N.  For few rows, of which a tile of 256 would be mostly empty and whose epilogue
// only the warps of their lanes could do: 9 rows of 114316 words at 168 36 -> 24 us, and
// for some hundred rows that tiles of 256 fit badly.
constexpr int kSwapRows = 896, kSwapAlways = 128, kSwapWidth = 512, kSwapStages = 8;
// the rows' references, factors and labels, at the ring's end
constexpr int kRowData = kSwapRows * 12;
constexpr int kOperandBytes = kHalf * kDepth * 2;
constexpr int kStageBytes = 2 * kOperandBytes;
// (with room for the rows' data behind as many stages: 7 for tiles of 160 rows)
constexpr int kRingBytes = kStages * kStageBytes + 1024;
// A warp's 32 rows x 64 columns of bf16 on their way out by TMA (128-byte swizzle).
constexpr int kOutBytes = 32 * 128;
constexpr int kEpiWarps = 8, kGemmThreads = 64 + 32 * kEpiWarps;
// Warps of the dW product that meanwhile join dh's splits: memory work beside the
// tensor cores' (join: the number of pairs that dh's product ran with, 0: none).
constexpr int kJoinThreads = 128;
constexpr int kMostPairs = kSms / 2;
// Tiles of partial sums of dh: splits of the vocabulary are made while they fit.
constexpr int kMostSplits = 96, kSplitTiles = 8 * kMostPairs;
constexpr float kFloor = -FLT_MAX;  // stands in for -inf as a maximum

enum Mode { kForward, kNumerators, kGradHidden, kGradWeight };
enum Word { kLive = 0, kArrived = 1, kErr = kCtrlErr };

struct Layout {
  int rows_pad, chunk, chunks, vocab_tiles, hidden_tiles, split_tiles;
  int rows_tile;  // swapped_rows()
  int64_t cells_stride;
  size_t ctrl, counts, orig, label, target, ref, unbias, scale, flags, rows, scaled, sums, cells, splits, acc, total;
};

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// bf16 parts of a scaled row in dW's contraction.  Its product with the label's exact
// numerator is most of a row of dW, so that its rounding is most of dW's error.  Up to
// 128 rows, where dW's product waits for memory, a second part holds the rest (for 64
// rows of 32000 words at 1024 dW's error against 64 bits 0.0023 -> 0.0017, its rounding to
// bf16 alone).  Above, it would double a product that the tensor cores bound: 1021 x 65537
// at 2048 478 -> 593 us, 4096 x 131072 3.11 -> 4.1 ms, for 0.0023 -> 0.0017 in bf16 and 0.0016
// -> 4e-5 in fp32; a bf16 program's dz is rounded alike.  (One rule for both types: dW in
// bf16 is the fp32 one rounded.)
__host__ __device__ inline int scaled_parts(int rows) { return rows <= 128 ? 2 : 1; }

// N of the products with swapped roles, or 0: rows are M, in tiles of 256.  The swapped
// epilogue takes twice the instructions: products along short rows keep the others
// unless they have few of them.
int swapped_rows(int rows, int hidden) {
  if (rows > kSwapRows) return 0;
  const int tiles = ceil_div(rows, kTile), n = ceil_div(ceil_div(rows, tiles), 32) * 32;
  if (rows <= kSwapAlways) return n < 64 ? 64 : n;
  return hidden >= kSwapWidth && n <= kTile * 7 / 8 ? n : 0;
}

Layout make_plan(int rows, int hidden, int vocab, bool grad_hidden, bool grad_weight) {
  Layout l;
  const bool grad = grad_hidden || grad_weight;
  l.rows_tile = swapped_rows(rows, hidden);
  const int rows_tile = l.rows_tile ? l.rows_tile : kTile;
  l.rows_pad = ceil_div(rows, kTile) * kTile;
  l.vocab_tiles = ceil_div(vocab, kTile);
  l.hidden_tiles = ceil_div(hidden, kTile);
  l.cells_stride = align_up((size_t)vocab, 64);
  // (the forward pass keeps 16 bytes for each row and 256 columns)
  int64_t most = grad ? kMostCells / l.cells_stride : ((int64_t)1 << 23) / l.vocab_tiles;
  most = most / kTile * kTile;
  if (most < kTile) most = kTile;
  l.chunk = most < l.rows_pad ? (int)most : l.rows_pad;
  l.chunks = ceil_div(l.rows_pad, l.chunk);
  l.split_tiles = 0;
  if (grad_hidden)
    for (int m = 1; m <= ceil_div(l.chunk, rows_tile); ++m) {
      const int tiles = m * l.hidden_tiles, kb = ceil_div(vocab, kDepth);
      int s = kSplitTiles / tiles;
      s = s < 1 ? 1 : s > kMostSplits ? kMostSplits : s;
      s = s < kb ? s : kb;
      if (s * tiles > l.split_tiles) l.split_tiles = s * tiles;
    }
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t r = o;
    o = align_up(o + bytes, 1024);
    return r;
  };
  const size_t n = (size_t)l.rows_pad;
  l.ctrl = take(kCtrlWords * 4);
  l.counts = take((n + 1023) / 1024 * 4);
  l.orig = take(n * 4);
  l.label = take(n * 4);
  l.target = take(n * 4);
  l.ref = take(n * 4);
  l.unbias = take(n * 4);
  l.scale = take(n * 4);
  l.flags = take(n / kTile * 3 * 4);
  l.rows = take(n * hidden * 2);
  l.scaled = take(grad_weight ? (size_t)l.chunk * scaled_parts(rows) * hidden * 2 : 0);
  l.sums = take((size_t)l.vocab_tiles * 2 * l.chunk * sizeof(float2));
  l.cells = take(grad ? (size_t)l.chunk * l.cells_stride * 2 : 0);
  l.splits = take((size_t)l.split_tiles * kTile * kTile * 4);
  l.acc = take(grad_weight && l.chunks > 1 ? (size_t)vocab * hidden * 4 : 0);
  l.total = o;
  return l;
}

// Device view of the workspace and the call.
struct Call {
  int T, H, V;
  float dense;  // given_back() of rows without a piece of zeros
  int rows_pad, chunk, vocab_tiles, hidden_tiles;
  int rows_tile;  // of the first product and dh's
  int64_t cells_stride;
  int32_t *ctrl, *orig, *label;
  int32_t *counts;  // labelled rows of each 1024 (more than kCountedRows rows)
  int32_t *flags;  // [3][rows_pad / 256]: tiles to run again; their list; each chunk's number of them
  float *target, *ref, *scale;
  float *unbias;  // of a row's logits: 1 + kTruncated for each element that is added
  __nv_bfloat16 *rows, *scaled, *cells;
  float2 *sums;   // [2 vocab_tiles][chunk]: sum of numerators, largest logit
  float *splits;  // [tiles][256][256]
  float *acc;     // [V][H], more than one chunk
  const __nv_bfloat16 *hidden, *weight;
  int64_t hidden_stride, weight_stride;
  const int32_t *labels;
  const float *row_weight;
  float *row_loss, *loss;
  __nv_bfloat16 *dh;
  int64_t dh_stride;
  void *dw;
  int dw_fp32;
  int64_t dw_stride;
};

__device__ __forceinline__ int chunk_rows(const Call &c, int chunk) {
  const int left = __ldcg(c.ctrl + kLive) - chunk * c.chunk;
  return left < 0 ? 0 : left < c.chunk ? left : c.chunk;
}

// Splits of dh's contraction: the fewest steps of 64 for the busiest pair, with a
// tile's accumulators and its share of the joining pass counted as steps.  By one
// warp, known to all its lanes.
__device__ __forceinline__ int choose_splits(int tiles, int kb, int pairs) {
  const int lane = threadIdx.x & 31;
  int most = kSplitTiles / tiles;
  most = max(1, min(min(most, kMostSplits), kb));
  uint32_t best = ~0u;
  for (int s = 1 + lane; s <= most; s += 32) {
    const uint32_t steps = (uint32_t)((tiles * s + pairs - 1) / pairs) * ((kb + s - 1) / s + 3) +
                           (uint32_t)(tiles * s) / 3;
    best = min(best, steps << 7 | (uint32_t)s);
  }
  return (int)(__reduce_min_sync(0xFFFFFFFFu, best) & 127u);
}

// ---------------------------------------------------------------------------
// rows with a label, moved together
// ---------------------------------------------------------------------------
constexpr int kGatherThreads = 256, kGatherRows = kGatherThreads / 32;
// More rows than this: the labels of each 1024 are counted first, and a CTA adds up
// counts instead of reading all labels before its own.
constexpr int kCountedRows = 8192;

__global__ void __launch_bounds__(1024) count_kernel(Call c) {
  pdl_launch_dependents();
  const int t = blockIdx.x * 1024 + threadIdx.x;
  const int n = __syncthreads_count(t < c.T && __ldg(c.labels + t) >= 0);
  if (threadIdx.x == 0) c.counts[blockIdx.x] = n;
}

// A warp a row: with a label, the row is copied to its place among those and its
// label's logit computed (fp32 sums of a lane's products, then over the lanes);
// without, it gets its results.
__global__ void __launch_bounds__(kGatherThreads, 2) gather_kernel(Call c, int counted) {
  __shared__ int before_all, in_warp[kGatherRows];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t0 = blockIdx.x * kGatherRows, t = t0 + warp;
  if (threadIdx.x == 0) before_all = 0;
  __syncthreads();
  pdl_wait_primary();
  pdl_launch_dependents();
  if (blockIdx.x == 0) {
    if (threadIdx.x != kLive && threadIdx.x < kCtrlWords) c.ctrl[threadIdx.x] = 0;
    for (int i = threadIdx.x; i < c.rows_pad / kTile * 3; i += kGatherThreads) c.flags[i] = 0;
  }
  // labelled rows before the CTA's, in whole numbers
  int n = 0;
  const int from = counted ? t0 / 1024 * 1024 : 0;
  if (counted)
    for (int i = threadIdx.x; i < from / 1024; i += kGatherThreads) n += __ldcg(c.counts + i);
#pragma unroll 8
  for (int i = from + threadIdx.x; i < t0; i += kGatherThreads) n += __ldg(c.labels + i) >= 0 ? 1 : 0;
  n = __reduce_add_sync(0xFFFFFFFFu, n);
  if (lane == 0 && n) atomicAdd(&before_all, n);
  const int y = t < c.T ? __ldg(c.labels + t) : -1;
  if (lane == 0) in_warp[warp] = y >= 0 ? 1 : 0;
  __syncthreads();
  const uint32_t live = __ballot_sync(0xFFFFFFFFu, lane < kGatherRows && in_warp[lane % kGatherRows] != 0);
  const int at = before_all + __popc(live & ((1u << warp) - 1));
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) c.ctrl[kLive] = before_all + __popc(live);
  if (t >= c.T) return;
  const int words = c.H / 8;
  if (y >= 0) {
    const uint4 *row = reinterpret_cast<const uint4 *>(c.hidden + (int64_t)t * c.hidden_stride);
    const bool known = y < c.V;
    const uint4 *head = reinterpret_cast<const uint4 *>(c.weight + (int64_t)(known ? y : 0) * c.weight_stride);
    uint4 *to = reinterpret_cast<uint4 *>(c.rows + (int64_t)at * c.H);
    float s = 0.0f;
    int added = 0;  // pieces that are not all zeros
#pragma unroll 4
    for (int k = lane; k < words; k += 32) {
      const uint4 a = __ldg(row + k), b = __ldg(head + k);
      to[k] = a;
      added += ((a.x | a.y | a.z | a.w) & 0x7FFF7FFFu) != 0u ? 1 : 0;
      const uint32_t av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        s = fmaf(__uint_as_float(av[q] << 16), __uint_as_float(bv[q] << 16), s);
        s = fmaf(__uint_as_float(av[q] & 0xFFFF0000u), __uint_as_float(bv[q] & 0xFFFF0000u), s);
      }
    }
    s = warp_sum(s);
    added = __reduce_add_sync(0xFFFFFFFFu, added);
    if (!known) s = __int_as_float(0x7FC00000);  // a label outside the vocabulary: NaN
    if (lane == 0) {
      c.unbias[at] = given_back(8 * added);
      c.orig[at] = t;
      c.label[at] = y;
      c.target[at] = c.ref[at] = s;
    }
  } else {
    if (lane == 0) c.row_loss[t] = 0.0f;
    if (c.dh) {
      uint4 *row = reinterpret_cast<uint4 *>(c.dh + (int64_t)t * c.dh_stride);
      for (int k = lane; k < words; k += 32) row[k] = make_uint4(0, 0, 0, 0);
    }
  }
}

// ---------------------------------------------------------------------------
// the products
// ---------------------------------------------------------------------------
struct Operands {
  CUtensorMap a, b;
  CUtensorMap out;  // bf16 results, boxes of 64 columns and 32 rows
};

// Shared-memory descriptor of an MN-major operand with 128-byte swizzle: groups
// of 64 elements across the contraction (128 bytes), `group` bytes apart, each of
// 8-deep blocks of 1024 bytes along it.
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t saddr, uint32_t group) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(group >> 4) << 16;  // leading: to the next 64 elements
  d |= (uint64_t)(1024 >> 4) << 32;   // stride: to the next 8 of the contraction
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// 32 accumulator columns of the thread's lane.
__device__ __forceinline__ void tmem_ld_row(uint32_t taddr, float (&v)[32]) {
  uint32_t *r = reinterpret_cast<uint32_t *>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
        "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
        "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]),
        "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// A warp's 64 columns of 32 rows, two to a word, from the buffer of its lanes' rows.
struct OutBuffer {
  uint32_t at;  // shared address, 1024-byte aligned
  // columns 32 h.. of this lane's row (h = 0, 1)
  __device__ __forceinline__ void put(int lane, int h, const uint32_t (&w)[16]) const {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(
                       at + (uint32_t)(lane * 128 + (((4 * h + c) ^ (lane & 7)) << 4))),
                   "r"(w[4 * c]), "r"(w[4 * c + 1]), "r"(w[4 * c + 2]), "r"(w[4 * c + 3])
                   : "memory");
  }
  // before it is written again: the last store has read it
  __device__ __forceinline__ void wait(int lane) const {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
  }
  __device__ __forceinline__ void send(int lane, const CUtensorMap *map, int x, int y) const {
    fence_proxy_async_shared();
    __syncwarp();
    if (lane == 0) {
      asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                       (uint64_t)map),
                   "r"(x), "r"(y), "r"(at)
                   : "memory");
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
  __device__ __forceinline__ void finish(int lane) const {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
};

struct Unit {
  int m, n, k0, k1;
};

template <Mode kMode>
struct Work {
  int mt, nt, kb, splits, units;
  const int *list;  // kNumerators again: the tiles of rows to take
  __device__ __forceinline__ Unit at(int u) const {
    Unit r;
    if constexpr (kMode == kForward || kMode == kNumerators) {
      // the row tiles of a column tile next to each other: the head is read once
      r.n = u / mt;
      r.m = u - r.n * mt;
      if (kMode == kNumerators && list) r.m = __ldcg(list + r.m);
      r.k0 = 0;
      r.k1 = kb;
    } else if constexpr (kMode == kGradHidden) {
      const int tiles = mt * nt, s = u / tiles, t = u - s * tiles;
      r.m = t / nt;
      r.n = t - r.m * nt;
      r.k0 = (int)((int64_t)kb * s / splits);
      r.k1 = (int)((int64_t)kb * (s + 1) / splits);
    } else {
      r.m = u / nt;
      r.n = u - r.m * nt;
      r.k0 = 0;
      r.k1 = kb;
    }
    return r;
  }
};

constexpr size_t kBars = (size_t)kRingBytes + kEpiWarps * kOutBytes;
// barriers, words, alignment
constexpr int kWords = 8 * (2 * kSwapStages + 5);
constexpr size_t kGemmSmem = kBars + kWords + 64 + 1024;

// Sums of the columns' numerators and the P tile of 32 columns.
template <Mode kMode>
__device__ __forceinline__ void numerators(const float (&z)[32], float unbias, float ref, int label, int valid,
                                           float &sum, float &most, uint32_t (&packed)[16]) {
  // label: the label's column here, or outside 0..31; valid: columns of the vocabulary
  const bool plain = __all_sync(0xFFFFFFFFu, (unsigned)label >= 32u) && valid >= 32;
  if constexpr (kMode == kForward) {
    float m = most;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      if (plain || (j < valid && j != label)) m = fmaxf(m, z[j]);
    }
    sum *= ex2((most - m) * kLog2e);
    most = m;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const float e = ex2(fmaf(z[j], unbias, -m) * kLog2e);
      if (plain || (j < valid && j != label)) s[j & 3] += e;
    }
    sum += (s[0] + s[1]) + (s[2] + s[3]);
  } else {
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
      float e[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        e[q] = ex2(fmaf(z[j + q], unbias, -ref) * kLog2e);
        if (plain || (j + q < valid && j + q != label)) {
          s[(j + q) & 3] += e[q];
          most = fmaxf(most, z[j + q]);
        }
      }
      packed[j / 2] = pack_bf16(e[0], e[1]);
    }
    sum += (s[0] + s[1]) + (s[2] + s[3]);
  }
}

__device__ __forceinline__ float warp_max_redux(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// 32 values of each lane reduced over the lanes: lane j gets value j's result.
template <typename F>
__device__ __forceinline__ float reduce_across(float (&x)[32], int lane, F op) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    const bool hi = (lane & o) != 0;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float other = __shfl_xor_sync(0xFFFFFFFFu, hi ? x[i] : x[i + o], o);
      x[i] = op(hi ? x[i + o] : x[i], other);
    }
  }
  return x[0];
}

// Swapped roles: 32 rows' logits z at the lane's word; unbias: their common factor.  Leaves
// their numerators in bf16 at `staged` (64 bytes a row, zeros for rows past `live`), and
// returns to lane j row j's sum over the warp's words and largest logit.
template <Mode kMode>
__device__ __forceinline__ float2 swapped_numerators(float (&z)[32], float unbias, const float *ref, const int *label, int word,
                                                 bool known, int live, int lane, uint32_t staged) {
  float top = kFloor;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const bool in = known && word != label[j];
    const float most = warp_max_redux(in ? z[j] : kFloor);
    if (lane == j) top = most;
    const float r = kMode == kForward ? most : ref[j];
    const float e = ex2(fmaf(z[j], unbias, -r) * kLog2e);
    if constexpr (kMode == kNumerators) {
      const __nv_bfloat16 h = __float2bfloat16_rn(j < live ? e : 0.0f);
      asm volatile("st.shared.b16 [%0], %1;" ::"r"(staged + (uint32_t)(j * 64 + lane * 2)),
                   "h"(*reinterpret_cast<const unsigned short *>(&h))
                   : "memory");
    }
    z[j] = in ? e : 0.0f;
  }
  const float sum = reduce_across(z, lane, [](float a, float b) { return a + b; });
  return make_float2(sum, top);
}

// Whether all threads of the epilogue say so (one that gave up takes the others along).
__device__ __forceinline__ bool epilogue_agrees(bool ok) {
  int r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.and.pred q, 2, %2, p;\n\t"
      "selp.s32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(ok ? 1 : 0), "n"(32 * kEpiWarps)
      : "memory");
  return r != 0;
}

// The loss over all rows, by N threads of a CTA: thread i adds its rows i, i + N, ...
// in fp64 and in order, then a butterfly and the warps in turn.  Rows without a label
// stay out whatever their weights (1 / the number of labelled rows may be 1 / 0).
template <int N>
__device__ __forceinline__ void total_loss(const Call &c, int thread, double *warps) {
  double s = 0.0;
#pragma unroll 4
  for (int t = thread; t < c.T; t += N) {
    const double l = (double)__ldcg(c.row_loss + t) * (c.row_weight ? (double)__ldg(c.row_weight + t) : 1.0);
    s += __ldg(c.labels + t) >= 0 ? l : 0.0;
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if ((thread & 31) == 0) warps[thread / 32] = s;
  asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory");
  if (thread == 0) {
    for (int w = 1; w < N / 32; ++w) s += warps[w];
    *c.loss = (float)s;
  }
}

// dh: the splits' sums of a row in order, times its factor; by `threads` threads, in
// whole warps.
__device__ __forceinline__ void join_rows(const Call &c, int chunk, int pairs, int64_t thread, int64_t threads) {
  const int rows = chunk_rows(c, chunk), row0 = chunk * c.chunk;
  if (rows == 0) return;
  const int tiles = (rows + c.rows_tile - 1) / c.rows_tile * c.hidden_tiles;
  const int splits = choose_splits(tiles, (c.V + kDepth - 1) / kDepth, pairs), words = c.H / 4;
  // four outputs at a time: their loads' latency is what this takes
  constexpr int kItems = 4;
  const int64_t all = (int64_t)rows * words;
  for (int64_t i0 = thread; i0 < all; i0 += kItems * threads) {
    const float *from[kItems];
    float4 v[kItems];
    int row[kItems], col[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int64_t i = i0 + k * threads < all ? i0 + k * threads : i0;
      row[k] = (int)(i / words);
      col[k] = (int)(i - (int64_t)row[k] * words) * 4;
      const int tile = row[k] / c.rows_tile * c.hidden_tiles + col[k] / kTile;
      from[k] = c.splits + ((int64_t)tile * kTile + row[k] % c.rows_tile) * kTile + col[k] % kTile;
      v[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
#pragma unroll 2
    for (int s = 0; s < splits; ++s) {
      float4 x[kItems];
#pragma unroll
      for (int k = 0; k < kItems; ++k) x[k] = __ldcg(reinterpret_cast<const float4 *>(from[k]));
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        v[k].x += x[k].x; v[k].y += x[k].y; v[k].z += x[k].z; v[k].w += x[k].w;
        from[k] += (int64_t)tiles * kTile * kTile;
      }
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      if (i0 + k * threads >= all) break;
      const float f = __ldcg(c.scale + row0 + row[k]);
      __nv_bfloat16 *to = c.dh + (int64_t)__ldcg(c.orig + row0 + row[k]) * c.dh_stride + col[k];
      *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(v[k].x * f, v[k].y * f), pack_bf16(v[k].z * f, v[k].w * f));
    }
  }
}

template <Mode kMode, bool kSwapped>
__global__ void __launch_bounds__(kGemmThreads + (kMode == kGradWeight ? kJoinThreads : 0), 1)
    product_kernel(const __grid_constant__ Operands maps, Call c, int chunk, int again, int join,
                   uint64_t timeout_ns) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char *smem = reinterpret_cast<unsigned char *>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t smem_base = smem_u32(smem);
  const uint32_t bar0 = smem_base + (uint32_t)kBars;
  // N, a stage of the ring, and how many there are
  const int n_rows = kSwapped ? c.rows_tile : kTile;
  const int slot_bytes = kSwapped ? kOperandBytes + n_rows * kDepth : kStageBytes;
  const int ring = kSwapped ? min(kSwapStages, (kRingBytes - kRowData) / slot_bytes) : kStages;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (ring + s); };
  auto accf_bar = [&](int b) { return bar0 + 8u * (2 * ring + b); };
  auto acce_bar = [&](int b) { return bar0 + 8u * (2 * ring + 2 + b); };
  const uint32_t drain_bar = bar0 + 8u * (2 * ring + 4);
  int *misc = reinterpret_cast<int *>(smem + kBars + kWords);
  volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(misc);
  volatile int *abort = misc + 1;
  volatile int *consumed = misc + 2;
  volatile int *n_splits = misc + 3;
  double *warp_totals = reinterpret_cast<double *>(misc + 4);  // kGradWeight
  float *row_ref = reinterpret_cast<float *>(smem + kRingBytes - kRowData);  // kSwapped
  float *row_unbias = row_ref + kSwapRows;
  int *row_label = reinterpret_cast<int *>(row_unbias + kSwapRows);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t crank = cluster_ctarank();
  const bool lead = crank == 0;
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  // (again: the first product's second run; dW's product behind the last chunk)
  // The second run has hardly ever anything to do: it looks first.
  // All others get ready while the kernel before ends.
  if (kMode == kNumerators && again) {
    pdl_wait_primary();
    if (__ldcg(c.flags + 2 * (c.rows_pad / kTile) + chunk) == 0) return;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < ring; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf_bar(b), 1);
      mbar_init(acce_bar(b), 2 * kEpiWarps);
    }
    mbar_init(drain_bar, 1);
    *abort = 0;
    *consumed = 0;
    mbar_fence_init();
    tma_prefetch_desc(&maps.a);
    tma_prefetch_desc(&maps.b);
    if constexpr (kMode == kNumerators && !kSwapped) tma_prefetch_desc(&maps.out);
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32((const void *)tmem_slot), 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  if (kMode != kNumerators || !again) pdl_wait_primary();
  const int rows = chunk_rows(c, chunk), row0 = chunk * c.chunk;
  Work<kMode> work;
  work.list = nullptr;
  work.splits = 1;
  if constexpr (kMode == kForward || kMode == kNumerators) {
    work.mt = (rows + n_rows - 1) / n_rows;
    work.nt = c.vocab_tiles;
    work.kb = (c.H + kDepth - 1) / kDepth;
    if (kMode == kNumerators && again) {
      // the tiles that the sums' kernel marked
      // (roles swapped: all rows, whose tiles are others)
      if constexpr (!kSwapped) {
        const int tiles = c.rows_pad / kTile;
        work.mt = __ldcg(c.flags + 2 * tiles + chunk);
        work.list = c.flags + tiles + row0 / kTile;
      }
    }
    work.units = work.mt * work.nt;
    if constexpr (kSwapped) {
      for (int i = threadIdx.x; i < work.mt * n_rows; i += blockDim.x) {
        row_ref[i] = i < rows ? __ldcg(c.ref + i) : 0.0f;
        row_unbias[i] = i < rows ? __ldcg(c.unbias + i) : c.dense;
        row_label[i] = i < rows ? __ldcg(c.label + i) : -1;
      }
      __syncthreads();
    }
  } else if constexpr (kMode == kGradHidden) {
    work.mt = (rows + n_rows - 1) / n_rows;
    work.nt = c.hidden_tiles;
    work.kb = (c.V + kDepth - 1) / kDepth;
    if (warp == 0 && rows > 0) {
      const int s = choose_splits(work.mt * work.nt, work.kb, pairs);
      if (lane == 0) *n_splits = s;
    }
    __syncthreads();
    work.splits = rows > 0 ? *n_splits : 0;
    work.units = work.mt * work.nt * work.splits;
  } else {
    work.mt = c.vocab_tiles;
    work.nt = c.hidden_tiles;
    work.kb = (rows + kDepth - 1) / kDepth * scaled_parts(c.T);
    work.units = rows > 0 ? work.mt * work.nt : 0;
    if (rows == 0 && chunk == 0) {
      // no labelled row at all: zeros (16 bytes are 8 elements, or 4)
      const int words = c.H / (c.dw_fp32 ? 4 : 8);
      const int64_t all = (int64_t)c.V * words;
      for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < all;
           i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t v = i / words, k = i - v * words;
        char *row = static_cast<char *>(c.dw) + v * c.dw_stride * (c.dw_fp32 ? 4 : 2);
        reinterpret_cast<uint4 *>(row)[k] = make_uint4(0, 0, 0, 0);
      }
    }
  }
  auto give_up = [&](int code) {
    if (!*abort) {
      *abort = 1;
      atomicOr(c.ctrl + kErr, code);
    }
  };
  if (threadIdx.x == 0 && !lead &&
      ld_shared_cluster(mapa_shared(smem_u32((const void *)tmem_slot), 0u)) != tmem_base)
    give_up(SLIMWISE_DEVERR_TMEM_PAIR);
  // a bounded wait of the warp: whether it completed on every lane
  auto all_ok = [&](bool ok) {
    if (!ok) give_up(SLIMWISE_DEVERR_PIPELINE_TIMEOUT);
    return __all_sync(0xFFFFFFFFu, ok) != 0;
  };
  // operands along the contraction (K-major) or across it
  constexpr bool kAcrossA = kMode == kGradWeight || (kSwapped && kMode == kGradHidden);
  constexpr bool kAcrossB = kMode == kGradWeight || (!kSwapped && kMode == kGradHidden);

  if (warp == 0) {
    // ------------------------------------------------------------ copies
    int stage = 0, issued = 0;
    uint32_t phase = 0;
    const uint64_t policy = l2_policy_evict_last();
    fence_proxy_async_global();  // what the kernels before stored is read by TMA
    bool ok = true;
    for (int u = pair; u < work.units && ok; u += pairs) {
      const Unit w = work.at(u);
      // first row (column) of this CTA's share of either operand
      const bool logits = kMode == kForward || kMode == kNumerators;
      const int a0 = (kSwapped ? w.n * kTile : (logits ? row0 : 0) + w.m * kTile) + (int)crank * kHalf;
      const int b0 = kSwapped ? w.m * n_rows + (int)crank * n_rows / 2 : w.n * kTile + (int)crank * kHalf;
      for (int k = w.k0; k < w.k1; ++k) {
        if (!all_ok(mbar_wait_bounded(empty_bar(stage), phase ^ 1u, abort, timeout_ns))) {
          ok = false;
          break;
        }
        const uint32_t a = smem_base + (uint32_t)(stage * slot_bytes), b = a + kOperandBytes;
        // (dW: the numerators again for the scaled rows' second part)
        const int half_k = kMode == kGradWeight && scaled_parts(c.T) > 1 ? work.kb / 2 : work.kb;
        const int ka = kMode == kGradWeight && k >= half_k ? k - half_k : k;
        const int kb_row = ka * kDepth + (ka != k ? c.chunk : 0);
        if (elect_one()) {
          const uint32_t bar = mapa_shared(full_bar(stage), 0u);
          if (lead)
            mbar_arrive_expect_tx(full_bar(stage), 2 * slot_bytes);
          if constexpr (kAcrossA) {
            tma_load_2d_pair(a, &maps.a, bar, a0, ka * kDepth, policy);
            tma_load_2d_pair(a + kOperandBytes / 2, &maps.a, bar, a0 + 64, ka * kDepth, policy);
          } else {
            tma_load_2d_pair(a, &maps.a, bar, k * kDepth, a0, policy);
          }
          if constexpr (kAcrossB) {
            tma_load_2d_pair(b, &maps.b, bar, b0, kb_row, policy);
            tma_load_2d_pair(b + kOperandBytes / 2, &maps.b, bar, b0 + 64, kb_row, policy);
          } else {
            tma_load_2d_pair(b, &maps.b, bar, k * kDepth, b0, policy);
          }
        }
        __syncwarp();
        ++issued;
        if (++stage == ring) {
          stage = 0;
          phase ^= 1u;
        }
      }
    }
    pdl_launch_dependents();
    if (lane == 0) {
      // until every stage still in the ring has been released (or, in the first
      // CTA after an abort, its copies have landed): nothing is left on its way
      // to this CTA's shared memory when it exits
      const int from = issued > ring ? issued - ring : 0;
      if (*abort && lead) {
        for (int s = *consumed > from ? *consumed : from; s < issued; ++s)
          mbar_wait_timeout(full_bar(s % ring), (uint32_t)((s / ring) & 1), 10000000ull);
      } else {
        for (int s = from; s < issued; ++s)
          mbar_wait_timeout(empty_bar(s % ring), (uint32_t)((s / ring) & 1), 10000000ull);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs
    if (lead) {
      int stage = 0, local = 0, n_consumed = 0;
      uint32_t phase = 0;
      const uint32_t idesc = idesc_bf16_f32(kTile, n_rows) | (kAcrossA ? 1u << 15 : 0u) |
                             (kAcrossB ? 1u << 16 : 0u);
      bool ok = true;
      for (int u = pair; u < work.units && ok; u += pairs, ++local) {
        const Unit w = work.at(u);
        const int b = local & 1;
        if (!all_ok(mbar_wait_cluster_bounded(acce_bar(b), ((uint32_t)(local >> 1) & 1u) ^ 1u, abort,
                                              timeout_ns)))
          break;
        tc_fence_after();
        const uint32_t d = tmem_base + (uint32_t)(b * kTile);
        for (int k = w.k0; k < w.k1; ++k) {
          if (!all_ok(mbar_wait_bounded(full_bar(stage), phase, abort, timeout_ns))) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t as = smem_base + (uint32_t)(stage * slot_bytes), bs = as + kOperandBytes;
          ++n_consumed;
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < kDepth / 16; ++kk)
              tc_mma_bf16_pair(d,
                               kAcrossA ? smem_desc_mn(as + kk * 2048, kOperandBytes / 2)
                                        : smem_desc_sw128(as + kk * 32),
                               kAcrossB ? smem_desc_mn(bs + kk * 2048, kOperandBytes / 2)
                                        : smem_desc_sw128(bs + kk * 32),
                               idesc, (k != w.k0 || kk != 0) ? 1u : 0u);
            tc_commit_pair(empty_bar(stage), (uint16_t)3);
            *consumed = n_consumed;
          }
          __syncwarp();
          if (++stage == ring) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (!ok) break;
        if (elect_one()) tc_commit_pair(accf_bar(b), (uint16_t)3);
        __syncwarp();
      }
      if (__any_sync(0xFFFFFFFFu, *abort != 0) && n_consumed > 0) {
        if (elect_one()) tc_commit_pair(drain_bar, (uint16_t)1);
        mbar_wait_timeout(drain_bar, 0, 10000000ull);
      }
    }
    __syncwarp();
  } else if (warp >= 2 + kEpiWarps) {
    // ------------------------------------------------------------ dh's splits
    // and, behind the last chunk, the loss
    if (join)
      join_rows(c, chunk, join, (int64_t)blockIdx.x * kJoinThreads + (threadIdx.x - kGemmThreads),
                (int64_t)gridDim.x * kJoinThreads);
    if (again && c.loss && blockIdx.x == 0) total_loss<kJoinThreads>(c, (int)threadIdx.x - kGemmThreads, warp_totals);
  } else {
    // ------------------------------------------------------------ accumulators
    const int q = warp & 3, half = (warp - 2) >> 2;  // lanes 32 q.., columns 128 half..
    const int in_tile = (int)crank * kHalf + 32 * q + lane;
    const OutBuffer out = {smem_base + (uint32_t)(kRingBytes + (warp - 2) * kOutBytes)};
    // kSwapped: the four warps' sums of a row, [2 tiles in turn][4][256], joined a tile later,
    // behind the barrier at which the warps agree on the next tile's wait
    float2 *quarters = reinterpret_cast<float2 *>(smem + kRingBytes + kEpiWarps * kOutBytes / 2);
    constexpr bool kSums = kSwapped && (kMode == kForward || kMode == kNumerators);
    Unit joined = {0, -1, 0, 0};
    auto join_quarters = [&](int parity) {
      const int t = threadIdx.x - 64, row = joined.m * n_rows + t;
      if (joined.n < 0 || t >= n_rows || row >= rows) return;
      const float2 *at = quarters + parity * 4 * kTile + t;
      float top = kFloor, sum = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k) top = fmaxf(top, at[k * kTile].y);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        sum += kMode == kForward ? at[k * kTile].x * ex2((at[k * kTile].y - top) * kLog2e) : at[k * kTile].x;
      c.sums[(int64_t)(joined.n * 2 + (int)crank) * c.chunk + row] = make_float2(sum, top);
    };
    int local = 0;
    for (int u = pair; u < work.units; u += pairs, ++local) {
      const Unit w = work.at(u);
      const int b = local & 1;
      bool ok = all_ok(mbar_wait_bounded(accf_bar(b), (uint32_t)(local >> 1) & 1u, abort, timeout_ns));
      if constexpr (kSums) {
        ok = epilogue_agrees(ok);
        join_quarters((local & 1) ^ 1);
        joined = w;
      }
      if (!ok) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(32 * q) << 16) + (uint32_t)(b * kTile + half * kHalf);
      const int row = w.m * kTile + in_tile, col0 = w.n * kTile + half * kHalf;
      auto release = [&]() {
        tc_fence_before();
        __syncwarp();
        // (relaxed: what it hands over is tensor memory, ordered by the fence above; a release
        // would wait for the tile before's stores)
        if (lane == 0)
          asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(
                           mapa_shared(acce_bar(b), 0u))
                       : "memory");
      };
      if constexpr (kSwapped) {
        // this lane's word of the vocabulary (dh: column), the tile's rows in 32s, which the
        // two halves of the warps take in turn
        const int mine = w.n * kTile + in_tile, row_first = w.m * n_rows;
        const uint32_t lanes = tmem_base + ((uint32_t)(32 * q) << 16) + (uint32_t)(b * kTile);
        const uint32_t staged = smem_base + (uint32_t)(kRingBytes + (warp - 2) * kOutBytes / 2);
#pragma unroll 1
        for (int t0 = 32 * half; t0 < n_rows; t0 += 64) {
          const int live = rows - row_first - t0;
          float z[32];
          tmem_ld_row(lanes + t0, z);
          tmem_ld_wait();
          if (t0 + 64 >= n_rows) release();
          if constexpr (kMode == kGradHidden) {
            float *to = c.splits + ((int64_t)u * kTile + t0) * kTile + in_tile;
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j < live) to[j * kTile] = z[j];
          } else {
            // (rows that are not dense: in advance, which rounds the logits once more.  Factors that
            // are read row by row in all cases cost 3 % of the product.)
            const float *unbias = row_unbias + row_first + t0;
            const bool dense = __all_sync(0xFFFFFFFFu, unbias[lane] == c.dense);
            if (!dense)
#pragma unroll
              for (int j = 0; j < 32; ++j) z[j] *= unbias[j];
            quarters[((local & 1) * 4 + q) * kTile + t0 + lane] =
                swapped_numerators<kMode>(z, dense ? c.dense : 1.0f, row_ref + row_first + t0, row_label + row_first + t0,
                                          mine, mine < c.V, live, lane, staged);
          }
          if constexpr (kMode == kNumerators) {
            // the warp's 32 words of each row, 64 bytes; as far as dW's slices read
            __syncwarp();
            const int first = w.n * kTile + (int)crank * kHalf + 32 * q;
            const int needed = (rows + kDepth - 1) / kDepth * kDepth - row_first - t0;
#pragma unroll
            for (int i = lane; i < 128; i += 32) {
              const int v = first + (i & 3) * 8;
              const uint4 x = ld_shared_v4(staged + (uint32_t)i * 16);
              if (v < c.cells_stride && (i >> 2) < needed)
                *reinterpret_cast<uint4 *>(c.cells + (int64_t)(row_first + t0 + (i >> 2)) * c.cells_stride + v) = x;
            }
            __syncwarp();
          }
        }
        // (a half without a 32 of its own)
        if (32 * half >= n_rows) release();
        if constexpr (kMode == kNumerators) {
          // zeros between the last tile and the end of dW's slices, which may lie further
          const int covered = row_first + n_rows, end = (rows + kDepth - 1) / kDepth * kDepth;
          if (half == 0 && w.m == work.mt - 1)
            for (int i = lane; i < (end - covered) * 4; i += 32) {
              const int v = w.n * kTile + (int)crank * kHalf + 32 * q + (i & 3) * 8;
              if (v < c.cells_stride)
                *reinterpret_cast<uint4 *>(c.cells + (int64_t)(covered + (i >> 2)) * c.cells_stride + v) =
                    make_uint4(0, 0, 0, 0);
            }
        }
      } else if constexpr (kMode == kForward || kMode == kNumerators) {
        // nothing reads what rows past the last one, rounded up to dW's slices, would leave
        if (row - lane >= (rows + kDepth - 1) / kDepth * kDepth) {
          release();
          continue;
        }
        const bool live = row < rows;
        const float ref = live ? __ldcg(c.ref + row0 + row) : 0.0f;
        const int label = live ? __ldcg(c.label + row0 + row) : -1;
        const float unbias = live ? __ldcg(c.unbias + row0 + row) : 1.0f;
        float sum = 0.0f, most = kFloor;
#pragma unroll 1
        for (int k = 0; k < kHalf / 32; ++k) {
          float z[32];
          uint32_t packed[16];
          tmem_ld_row(taddr + k * 32, z);
          tmem_ld_wait();
          if (k == kHalf / 32 - 1) release();
          const int col = col0 + 32 * k;
          numerators<kMode>(z, unbias, ref, label - col, c.V - col, sum, most, packed);
          if constexpr (kMode == kNumerators) {
            // rows past the last one: zeros (they are in the contraction of dW)
            if (!live)
#pragma unroll
              for (int j = 0; j < 16; ++j) packed[j] = 0u;
            if ((k & 1) == 0) out.wait(lane);
            out.put(lane, k & 1, packed);
            if ((k & 1) && col - 32 < c.cells_stride) out.send(lane, &maps.out, col - 32, row - lane);
          }
        }
        c.sums[(int64_t)(w.n * 2 + half) * c.chunk + row] = make_float2(sum, most);
      } else if constexpr (kMode == kGradHidden) {
        if (row - lane >= rows) {
          release();
          continue;
        }
        float *to = c.splits + ((int64_t)u * kTile + in_tile) * kTile + half * kHalf;
#pragma unroll 1
        for (int k = 0; k < kHalf / 32; ++k) {
          float z[32];
          tmem_ld_row(taddr + k * 32, z);
          tmem_ld_wait();
          if (k == kHalf / 32 - 1) release();
          if (row < rows && col0 + 32 * k < c.H)
#pragma unroll
            for (int j = 0; j < 32; j += 4)
              *reinterpret_cast<float4 *>(to + 32 * k + j) = make_float4(z[j], z[j + 1], z[j + 2], z[j + 3]);
        }
      } else {
        // chunks before the last leave fp32 sums; the last one adds them and rounds
        const bool last = __ldcg(c.ctrl + kLive) <= row0 + c.chunk;
        float *acc = c.acc + (int64_t)row * c.H;
#pragma unroll 1
        for (int k = 0; k < kHalf / 32; ++k) {
          float z[32];
          tmem_ld_row(taddr + k * 32, z);
          tmem_ld_wait();
          if (k == kHalf / 32 - 1) release();
          const int col = col0 + 32 * k;
          if (chunk > 0 && row < c.V)
#pragma unroll
            for (int j = 0; j < 32; j += 4)
              if (col + j < c.H) {
                const float4 x = __ldcg(reinterpret_cast<const float4 *>(acc + col + j));
                z[j] += x.x; z[j + 1] += x.y; z[j + 2] += x.z; z[j + 3] += x.w;
              }
          if (last && !c.dw_fp32) {
            uint32_t packed[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) packed[j] = pack_bf16(z[2 * j], z[2 * j + 1]);
            if ((k & 1) == 0) out.wait(lane);
            out.put(lane, k & 1, packed);
            if ((k & 1) && col - 32 < c.H && row - lane < c.V) out.send(lane, &maps.out, col - 32, row - lane);
          } else if (row < c.V) {
            float *to = last ? static_cast<float *>(c.dw) + (int64_t)row * c.dw_stride : acc;
#pragma unroll
            for (int j = 0; j < 32; j += 4)
              if (col + j < c.H)
                *reinterpret_cast<float4 *>(to + col + j) = make_float4(z[j], z[j + 1], z[j + 2], z[j + 3]);
          }
        }
      }
    }
    out.finish(lane);
    if constexpr (kSums) {
      if (epilogue_agrees(!*abort)) join_quarters((local & 1) ^ 1);
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

// ---------------------------------------------------------------------------
// a row's sums
// ---------------------------------------------------------------------------
// Eight rows a CTA; the column tiles' sums of a row in 32 parts, four in a warp.  kForward: the
// loss.  kNumerators: besides, the row's factor, the label's numerator and the
// scaled row; `again`: only rows of the tiles that were run again (roles swapped: all; else a row whose
// reference does not do marks its tile).
constexpr int kSumRows = 8, kSumThreads = 32 * kSumRows;

template <Mode kMode>
__global__ void __launch_bounds__(kSumThreads, 2) sums_kernel(Call c, int chunk, int again, int finish) {
  __shared__ float part_sum[32][kSumRows + 1], part_most[32][kSumRows + 1];
  __shared__ double total[kSumThreads / 32];
  __shared__ int last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait_primary();
  pdl_launch_dependents();
  if (again && __ldcg(c.flags + 2 * (c.rows_pad / kTile) + chunk) == 0) return;
  const int rows = chunk_rows(c, chunk), row0 = chunk * c.chunk;
  const int first = blockIdx.x * kSumRows, tile = row0 / kTile + first / kTile;
  const bool mine = first < (rows + kTile - 1) / kTile * kTile && (!again || c.rows_tile != kTile || __ldcg(c.flags + tile) != 0);
  if (mine) {
    // a warp's row and what is known of it
    const int row = first + warp, at = row0 + row;
    const bool live = row < rows;
    const float z = live ? __ldcg(c.target + at) : 0.0f;
    float ref = live ? __ldcg(c.ref + at) : 0.0f;
    const int t = live ? __ldcg(c.orig + at) : 0, y = live ? __ldcg(c.label + at) : -1;
    const float weight = live && c.row_weight ? __ldg(c.row_weight + t) : 1.0f;
    // every 32nd part of a row
    const int mine_row = lane & (kSumRows - 1), share = warp * (32 / kSumRows) + lane / kSumRows;
    const int parts = c.vocab_tiles * 2;
    float s = 0.0f, m = kFloor;
    const float2 *part = c.sums + first + mine_row;
#pragma unroll 8
    for (int i = share; i < parts; i += 32) {
      const float2 v = __ldcg(part + (int64_t)i * c.chunk);
      if constexpr (kMode == kForward) {
        const float to = fmaxf(m, v.y);
        s = s * ex2((m - to) * kLog2e) + v.x * ex2((v.y - to) * kLog2e);
        m = to;
      } else {
        s += v.x;
        m = fmaxf(m, v.y);
      }
    }
    part_sum[share][mine_row] = s;
    part_most[share][mine_row] = m;
    __syncthreads();
    float S = part_sum[lane][warp], top = part_most[lane][warp];
    const float mine_most = top;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if constexpr (kMode == kForward) {
      ref = z != z ? z : fmaxf(top, z);
      S *= ex2((mine_most - ref) * kLog2e);
    }
    S = warp_sum(S);
    // a logit of +inf: the formula has no number, but the others' exponentials are 0 where it is the
    // label's, and the sum's inverse is 0 where it is another's.  Nor where the label's is the only
    // one and -inf.
    if (z == INFINITY || top == INFINITY || (z == -INFINITY && S == 0.0f)) S = __int_as_float(0x7FC00000);
    const float own = ref == z ? 1.0f : ex2((z - ref) * kLog2e);
    float scale = 0.0f;
    if (live) {
      if constexpr (kMode == kNumerators) {
        // -S is the largest numerator: its rounding goes into the row's factor, and so to
        // the others, whose products with the operands mostly cancel
        const __nv_bfloat16 least = __float2bfloat16_rn(-S);
        const float ratio = S / -__bfloat162float(least);
        scale = weight / (own + S) * (ratio > 0.5f && ratio < 2.0f ? ratio : 1.0f);
        if (lane == 0) {
          c.scale[at] = scale;
          if (y < c.V) c.cells[(int64_t)row * c.cells_stride + y] = least;
          // (a label's logit of -inf: S is no number where another one is -inf too, unless all are)
          if (!again && (S > expf(kMostLoss) || (z == -INFINITY && top > kFloor && top < INFINITY))) {
            c.ref[at] = top;
            const int tiles = c.rows_pad / kTile;
            if (atomicExch(c.flags + tile, 1) == 0)
              c.flags[tiles + row0 / kTile + atomicAdd(c.flags + 2 * tiles + chunk, 1)] = tile - row0 / kTile;
          }
        }
      }
      if (lane == 0) c.row_loss[t] = ref == z ? log1pf(S) : (ref - z) + logf(own + S);
    }
    if constexpr (kMode == kNumerators) {
      if (c.scaled) {
        const uint4 *from = reinterpret_cast<const uint4 *>(c.rows + (int64_t)at * c.H);
        uint4 *to = reinterpret_cast<uint4 *>(c.scaled + (int64_t)row * c.H);
#pragma unroll 4
        for (int k = lane; k < c.H / 8; k += 32) {
          uint4 v = live ? __ldcg(from + k) : make_uint4(0, 0, 0, 0), rest;
          uint32_t *x = reinterpret_cast<uint32_t *>(&v), *y2 = reinterpret_cast<uint32_t *>(&rest);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float lo = __uint_as_float(x[q] << 16) * scale, hi = __uint_as_float(x[q] & 0xFFFF0000u) * scale;
            x[q] = pack_bf16(lo, hi);
            y2[q] = pack_bf16(lo - __uint_as_float(x[q] << 16), hi - __uint_as_float(x[q] & 0xFFFF0000u));
          }
          to[k] = v;
          if (scaled_parts(c.T) > 1) to[k + (int64_t)c.chunk * (c.H / 8)] = rest;
        }
      }
    }
  }
  if (!finish || !c.loss) return;
  // the forward pass: the CTA that ends last adds up the loss
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(c.ctrl + kArrived, 1) == (int)gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (last) total_loss<kSumThreads>(c, threadIdx.x, total);
}

// By itself where dW is not wanted.
__global__ void __launch_bounds__(256, 1) join_kernel(Call c, int chunk, int pairs, int finish) {
  __shared__ double warp_totals[8];
  pdl_wait_primary();
  pdl_launch_dependents();
  if (finish && c.loss && blockIdx.x == 0) total_loss<256>(c, threadIdx.x, warp_totals);
  join_rows(c, chunk, pairs, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
PFN_cuTensorMapEncodeTiled_v12000 encoder() {
  static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> fn{nullptr};
  PFN_cuTensorMapEncodeTiled_v12000 f = fn.load(std::memory_order_acquire);
  if (!f) {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) !=
            cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      return nullptr;
    f = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    fn.store(f, std::memory_order_release);
  }
  return f;
}

// A bf16 matrix of `rows` rows of `cols`, `stride` elements apart, in boxes of 64
// columns and `box` rows; 128-byte swizzle, zeros outside.
bool encode(CUtensorMap *map, const void *base, int64_t rows, int64_t cols, int64_t stride, int box) {
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
  cuuint32_t boxes[2] = {(cuuint32_t)kDepth, (cuuint32_t)box};
  cuuint32_t steps[2] = {1, 1};
  const auto f = encoder();
  return f && f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, boxes,
                steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Pairs that run at once (their CTAs' SMs lie in one cluster's reach); readies the
// kernel on the current device.
template <Mode kMode, bool kSwapped>
cudaError_t resident_pairs(int *pairs) {
  static std::atomic<int> known[64];
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  if (dev < 64 && (*pairs = known[dev].load(std::memory_order_acquire)) > 0) return cudaSuccess;
  auto kernel = product_kernel<kMode, kSwapped>;
  err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGemmSmem);
  if (err != cudaSuccess) return err;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2);
  cfg.blockDim = dim3(kGemmThreads + (kMode == kGradWeight ? kJoinThreads : 0));
  cfg.dynamicSmemBytes = kGemmSmem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  err = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
  if (err != cudaSuccess) return err;
  if (n < 1) return cudaErrorInvalidConfiguration;
  *pairs = n < kMostPairs ? n : kMostPairs;
  if (dev < 64) known[dev].store(*pairs, std::memory_order_release);
  return cudaSuccess;
}

template <Mode kMode, bool kSwapped = false>
cudaError_t run_product(const Operands &maps, const Call &c, int chunk, int again, int join, cudaStream_t stream,
                        int *used = nullptr) {
  constexpr int kThreads = kGemmThreads + (kMode == kGradWeight ? kJoinThreads : 0);
  int pairs = 0;
  const cudaError_t err = resident_pairs<kMode, kSwapped>(&pairs);
  if (err != cudaSuccess) return err;
  if (used) *used = pairs;
  return launch_chained(product_kernel<kMode, kSwapped>, dim3(2 * pairs), dim3(kThreads), kGemmSmem, stream, 2,
                        true, maps, c, chunk, again, join, kDefaultWaitLimitNs);
}

}  // namespace

size_t linear_loss_workspace(int rows, int hidden, int vocab, bool grad_hidden, bool grad_weight) {
  return make_plan(rows, hidden, vocab, grad_hidden, grad_weight).total;
}

cudaError_t launch_linear_loss(const LinearLossArgs &a, void *workspace, cudaStream_t stream) {
  const bool grad = a.grad_hidden || a.grad_weight;
  const Layout l = make_plan(a.rows, a.width, a.vocab, a.grad_hidden != nullptr, a.grad_weight != nullptr);
  char *w = static_cast<char *>(workspace);
  Call c = {};
  c.T = a.rows; c.H = a.width; c.V = a.vocab;
  c.dense = given_back(c.H);
  c.rows_pad = l.rows_pad; c.chunk = l.chunk;
  c.vocab_tiles = l.vocab_tiles; c.hidden_tiles = l.hidden_tiles;
  c.rows_tile = l.rows_tile ? l.rows_tile : kTile;
  c.cells_stride = l.cells_stride;
  c.ctrl = reinterpret_cast<int32_t *>(w + l.ctrl);
  c.counts = reinterpret_cast<int32_t *>(w + l.counts);
  c.orig = reinterpret_cast<int32_t *>(w + l.orig);
  c.label = reinterpret_cast<int32_t *>(w + l.label);
  c.flags = reinterpret_cast<int32_t *>(w + l.flags);
  c.target = reinterpret_cast<float *>(w + l.target);
  c.ref = reinterpret_cast<float *>(w + l.ref);
  c.unbias = reinterpret_cast<float *>(w + l.unbias);
  c.scale = reinterpret_cast<float *>(w + l.scale);
  c.rows = reinterpret_cast<__nv_bfloat16 *>(w + l.rows);
  c.scaled = a.grad_weight ? reinterpret_cast<__nv_bfloat16 *>(w + l.scaled) : nullptr;
  c.cells = reinterpret_cast<__nv_bfloat16 *>(w + l.cells);
  c.sums = reinterpret_cast<float2 *>(w + l.sums);
  c.splits = reinterpret_cast<float *>(w + l.splits);
  c.acc = reinterpret_cast<float *>(w + l.acc);
  c.hidden = static_cast<const __nv_bfloat16 *>(a.hidden);
  c.weight = static_cast<const __nv_bfloat16 *>(a.weight);
  c.hidden_stride = a.hidden_stride; c.weight_stride = a.weight_stride;
  c.labels = a.labels; c.row_weight = a.row_weight; c.row_loss = a.row_loss; c.loss = a.loss;
  c.dh = static_cast<__nv_bfloat16 *>(a.grad_hidden); c.dh_stride = a.grad_hidden_stride;
  c.dw = a.grad_weight; c.dw_fp32 = a.grad_weight_dtype == SLIMWISE_DTYPE_FP32; c.dw_stride = a.grad_weight_stride;

  Operands logits = {}, dh = {}, dw = {};
  // (rows past the call's are zeros without being read)
  const bool swapped = l.rows_tile > 0;
  const int half = c.rows_tile / 2;  // a CTA's rows of a tile
  bool ok = encode(swapped ? &logits.b : &logits.a, c.rows, c.T, c.H, c.H, half) &&
            encode(swapped ? &logits.a : &logits.b, c.weight, c.V, c.H, c.weight_stride, kHalf);
  if (grad && !swapped) ok = ok && encode(&logits.out, c.cells, l.chunk, l.cells_stride, l.cells_stride, 32);
  // (rows of the numerators past the call's, rounded up to dW's slices, are never written)
  const int cell_rows = ceil_div(c.T, kDepth) * kDepth < l.chunk ? ceil_div(c.T, kDepth) * kDepth : l.chunk;
  if (a.grad_hidden)  // e along the vocabulary, the head across it
    ok = ok && encode(swapped ? &dh.b : &dh.a, c.cells, cell_rows, c.V, l.cells_stride, half) &&
         encode(swapped ? &dh.a : &dh.b, c.weight, c.V, c.H, c.weight_stride, kDepth);
  if (a.grad_weight)  // both across the rows
    ok = ok && encode(&dw.a, c.cells, cell_rows, c.V, l.cells_stride, kDepth) &&
         encode(&dw.b, c.scaled, (int64_t)l.chunk * scaled_parts(c.T), c.H, c.H, kDepth) &&
         (c.dw_fp32 || encode(&dw.out, c.dw, c.V, c.H, c.dw_stride, 32));
  if (!ok) return cudaErrorInvalidValue;

  const int counted = c.T > kCountedRows;
  cudaError_t err = cudaSuccess;
  if (counted)
    err = launch_chained(count_kernel, dim3((unsigned)ceil_div(c.T, 1024)), dim3(1024), 0, stream, 1, false, c);
  if (err == cudaSuccess)
    err = launch_chained(gather_kernel, dim3((unsigned)ceil_div(c.T, kGatherRows)), dim3(kGatherThreads), 0, stream,
                         1, counted != 0, c, counted);
  for (int k = 0; k < l.chunks && err == cudaSuccess; ++k) {
    const dim3 sum_grid((unsigned)(l.chunk / kSumRows));
    const int finish = k == l.chunks - 1;
    if (!grad) {
      err = swapped ? run_product<kForward, true>(logits, c, k, 0, 0, stream)
                : run_product<kForward>(logits, c, k, 0, 0, stream);
      if (err == cudaSuccess)
        err = launch_chained(sums_kernel<kForward>, sum_grid, dim3(kSumThreads), 0, stream, 1, true, c, k, 0, finish);
      continue;
    }
    for (int again = 0; again < 2 && err == cudaSuccess; ++again) {
      err = swapped ? run_product<kNumerators, true>(logits, c, k, again, 0, stream)
                : run_product<kNumerators>(logits, c, k, again, 0, stream);
      if (err == cudaSuccess)
        err = launch_chained(sums_kernel<kNumerators>, sum_grid, dim3(kSumThreads), 0, stream, 1, true, c, k, again, 0);
    }
    int pairs = 0;
    if (a.grad_hidden && err == cudaSuccess) {
      err = swapped ? run_product<kGradHidden, true>(dh, c, k, 0, 0, stream, &pairs)
                : run_product<kGradHidden>(dh, c, k, 0, 0, stream, &pairs);
      if (err == cudaSuccess && !a.grad_weight)
        err = launch_chained(join_kernel, dim3(kSms * 8), dim3(256), 0, stream, 1, true, c, k, pairs, finish);
    }
    if (a.grad_weight && err == cudaSuccess) err = run_product<kGradWeight>(dw, c, k, finish, pairs, stream);
  }
  return err;
}

}  // namespace slimwise
