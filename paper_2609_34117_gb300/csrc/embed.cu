// embed.cu -- rows of an embedding table by token id, and the table's gradient.
//
//   out[i]    = scale table[id_i]           (id < 0: zeros; id >= vocab: NaN)
//   dtable[v] = scale sum over i with id_i = v of dout[i]
//
// Both move bytes: the lookup reads the rows asked for and writes them; the
// gradient reads dout once and writes the whole table, most of it zeros.
//
// The gradient's order of summation must not depend on timing, so there are no
// atomics on it.  One cluster sorts the positions by token (a stable radix sort
// in two or three passes, histograms in shared memory).  The next kernel sums the
// sorted rows in pieces of some positions: a token that lies inside a piece is
// written, one that crosses its border leaves fp32 sums, which a third kernel adds
// in order.  A token that occurs thousands of times is so spread over hundreds of
// CTAs.  Most of the time is the zeros of the tokens that do not occur.  CTAs of the second
// and third kernel write them, which find their tokens' presence by reading all ids
// and wait for no kernel: they run beside the sort, the sums and the joins.
#include "train.cuh"

namespace slimwise {

namespace {

// ---------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------
constexpr int kLookupThreads = 256, kLookupLoads = 8;

// A warp copies strips of kLookupLoads accesses a lane.
template <typename T, int V>
__global__ void __launch_bounds__(kLookupThreads)
    embed_kernel(const T *__restrict__ table, int vocab, int hidden, int64_t stride,
                 const int32_t *__restrict__ ids, int rows, float scale, T *__restrict__ out,
                 int64_t out_stride) {
  constexpr int E = V == 1 && sizeof(T) == 2 ? 2 * kLookupLoads : V * kLookupLoads;
  using Part = RowPart<T, V, E>;
  constexpr int kStrip = 32 * E;
  const int lane = threadIdx.x & 31;
  const int strips = (hidden + kStrip - 1) / kStrip;
  const int64_t all = (int64_t)rows * strips;
  const int64_t warps = (int64_t)gridDim.x * (kLookupThreads / 32);
  for (int64_t u = (int64_t)blockIdx.x * (kLookupThreads / 32) + (threadIdx.x >> 5); u < all; u += warps) {
    const int i = (int)(u / strips), c = (int)(u % strips) * kStrip;
    const int id = __ldg(ids + i);
    Part p;
    if (id >= 0 && id < vocab) {
      p.load(table + (int64_t)id * stride + c, lane, 32, hidden - c);
#pragma unroll
      for (int e = 0; e < E; e += 2) p.set2(e, p.get(e) * scale, p.get(e + 1) * scale);
    } else {
      const float v = id < 0 ? 0.0f : __int_as_float(0x7FC00000);
#pragma unroll
      for (int e = 0; e < E; e += 2) p.set2(e, v, v);
    }
    p.store(out + (int64_t)i * out_stride + c, lane, 32, hidden - c);
  }
}

// ---------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------
constexpr int kSortCtas = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
// Sorted positions that a group sums: enough pieces for all SMs where there are few,
// and, where there are many, pieces that keep the joins of a frequent token short.
constexpr int kLeastPiece = 4, kMostPiece = 256;
constexpr int kSumThreads = 256;

constexpr int kHalves = kSortThreads / kDigits;  // parts of the warps, in the sum over them
constexpr int kHeldItems = 4;                     // of a lane, read once a pass
static_assert(kSortWarps % kHalves == 0, "parts of the warps");
struct SortShared {
  uint32_t count[kSortWarps][kDigits];  // of a warp's items, then of those before it in its half
  uint32_t start[kHalves][kDigits];     // a half's items, then where they go
  uint32_t total[kDigits];              // of the CTA's items
  uint32_t scan[kDigits / 32];
};
// Bits of the largest key: vocab itself, the key of ids outside the table.
__host__ __device__ inline int key_bits(int vocab) {
  int b = 1;
  while (vocab >> b) ++b;
  return b;
}

// An item: x = key, y = position.  The last pass leaves them in a.
struct SortArgs {
  const int32_t *ids;
  int n, vocab;
  uint2 *a, *b;
};

__device__ __forceinline__ uint32_t cluster_load(const uint32_t *p, uint32_t rank) {
  return ld_shared_cluster(mapa_shared(smem_u32(p), rank));
}

// Lanes whose digit is this lane's, of those that have one: a ballot a bit (a
// match over the warp takes longer the more digits differ: 32768 ids 25 us with it).
__device__ __forceinline__ uint32_t lanes_with(uint32_t d) {
  uint32_t same = __ballot_sync(0xFFFFFFFFu, d < kDigits);
#pragma unroll
  for (int b = 0; b < kDigitBits; ++b) {
    const bool set = (d >> b & 1u) != 0;
    const uint32_t v = __ballot_sync(0xFFFFFFFFu, set);
    same &= set ? v : ~v;
  }
  return same;
}

// Stable sort by key, one cluster.  A warp holds a run of the items; the digits
// of its items are counted, counts become the warps' first places, digit by digit, and
// the items are moved in order.  Up to kHeldItems a lane they stay in registers between.
__device__ void sort_by_id(const SortArgs &s, SortShared &sh) {
  const int ctas = (int)gridDim.x, cta = (int)cluster_ctarank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int bits = key_bits(s.vocab), passes = (bits + kDigitBits - 1) / kDigitBits;
  const int width = (bits + passes - 1) / passes;
  // items of a warp, a multiple of 32
  const int per = ((s.n + ctas * kSortWarps - 1) / (ctas * kSortWarps) + 31) / 32 * 32;
  const int64_t first = (int64_t)(cta * kSortWarps + warp) * per;
  const int lo = (int)(first < s.n ? first : s.n), hi = (int)(first + per < s.n ? first + per : s.n);
  const int digit = threadIdx.x & (kDigits - 1), half = threadIdx.x / kDigits;
  constexpr int kPart = kSortWarps / kHalves, kBatch = 32 * kHeldItems;
  for (int pass = 0; pass < passes; ++pass) {
    // the last pass writes s.a
    const uint2 *src = (passes - pass) & 1 ? s.b : s.a;
    uint2 *dst = (passes - pass) & 1 ? s.a : s.b;
    const int shift = pass * width;
    uint2 held[kHeldItems];
    auto fetch = [&](int i0) {
#pragma unroll
      for (int k = 0; k < kHeldItems; ++k) {
        const int i = i0 + 32 * k + lane;
        held[k] = make_uint2(0u, 0u);
        if (i >= hi) continue;
        if (pass > 0) {
          held[k] = __ldcg(src + i);
        } else {
          const int id = __ldg(s.ids + i);
          held[k] = make_uint2(id >= 0 && id < s.vocab ? (uint32_t)id : (uint32_t)s.vocab, (uint32_t)i);
        }
      }
    };
    auto digit_of = [&](int k, int i0) {
      return i0 + 32 * k + lane < hi ? (held[k].x >> shift) & (kDigits - 1) : (uint32_t)kDigits;
    };
    fetch(lo);
    for (int i = threadIdx.x; i < kSortWarps * kDigits / 4; i += kSortThreads)
      reinterpret_cast<uint4 *>(&sh.count[0][0])[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    uint32_t alike[kHeldItems];  // of the held items: lanes of the same digit
    for (int i0 = lo; i0 < hi; i0 += kBatch) {
      if (i0 > lo) fetch(i0);
#pragma unroll
      for (int k = 0; k < kHeldItems; ++k) {
        if (i0 + 32 * k >= hi) break;
        const uint32_t d = digit_of(k, i0);
        const uint32_t same = alike[k] = lanes_with(d);
        if (d < kDigits && (same & ((1u << lane) - 1)) == 0) sh.count[warp][d] += __popc(same);
        __syncwarp();
      }
    }
    __syncthreads();
    {
      uint32_t c[kPart], sum = 0;
#pragma unroll
      for (int w = 0; w < kPart; ++w) c[w] = sh.count[half * kPart + w][digit];
#pragma unroll
      for (int w = 0; w < kPart; ++w) {
        sh.count[half * kPart + w][digit] = sum;
        sum += c[w];
      }
      sh.start[half][digit] = sum;
    }
    __syncthreads();
    uint32_t mine = 0;
    if (threadIdx.x < kDigits) {
#pragma unroll
      for (int h = 0; h < kHalves; ++h) mine += sh.start[h][digit];
      sh.total[digit] = mine;
    }
    uint32_t before = 0, all = mine;  // this digit's items in earlier CTAs, in all
    if (ctas > 1) {
      cluster_sync_all();
      if (threadIdx.x < kDigits) {
        all = 0;
        for (int c = 0; c < ctas; ++c) {
          const uint32_t v = cluster_load(&sh.total[digit], (uint32_t)c);
          before += c < cta ? v : 0u;
          all += v;
        }
      }
    }
    // exclusive scan of `all` over the digits
    uint32_t inc = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, inc, o);
      if (lane >= o) inc += v;
    }
    if (lane == 31 && threadIdx.x < kDigits) sh.scan[warp] = inc;
    __syncthreads();
    if (threadIdx.x < kDigits) {
      uint32_t base = before + inc - all;
      const uint32_t earlier = lane < warp ? sh.scan[lane] : 0u;  // (as many warps as lanes at the most)
      base += __reduce_add_sync(0xFFFFFFFFu, earlier);
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        const uint32_t n = sh.start[h][digit];
        sh.start[h][digit] = base;
        base += n;
      }
    }
    __syncthreads();
    for (int i0 = lo; i0 < hi; i0 += kBatch) {
      if (per > kBatch) fetch(i0);
#pragma unroll
      for (int k = 0; k < kHeldItems; ++k) {
        if (i0 + 32 * k >= hi) break;
        const uint32_t d = digit_of(k, i0);
        const uint32_t same = per > kBatch ? lanes_with(d) : alike[k];
        const uint32_t rank = __popc(same & ((1u << lane) - 1));
        const bool in = d < kDigits;
        const uint32_t place = in ? sh.start[warp / kPart][d] + sh.count[warp][d] + rank : 0u;
        __syncwarp();
        if (in) {
          dst[place] = held[k];
          if (rank == 0) sh.count[warp][d] += __popc(same);
        }
        __syncwarp();
      }
    }
    // the pass's items, written by all CTAs, are read by the next; totals are read no more
    if (ctas > 1) cluster_sync_all();
    else __syncthreads();
  }
}

__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(SortArgs s) {
  extern __shared__ __align__(16) unsigned char smem[];
  pdl_launch_dependents();
  sort_by_id(s, *reinterpret_cast<SortShared *>(smem));
}

// Zeros for the tokens of [from, to) that do not occur: the share of CTA `cta` of
// `ctas`, kSumThreads threads each.
constexpr int kZeroCtas = 2 * kSms, kZeroRows = 4096;
struct ZeroArgs {
  const int32_t *ids;
  int ctas, from, to;  // 0 CTAs: none
};
template <typename O>
__device__ void write_zeros(const ZeroArgs &z, int n, int hidden, O *out, int64_t out_stride) {
  __shared__ uint32_t present[kZeroRows / 32];
  const int lane = threadIdx.x & 31, per = (z.to - z.from + z.ctas - 1) / z.ctas;
  const int64_t first = z.from + (int64_t)blockIdx.x * per;
  const int end_row = (int)(first + per < z.to ? first + per : z.to);
  for (int lo = (int)first; lo < end_row; lo += kZeroRows) {
    const int rows = min(kZeroRows, end_row - lo);
    __syncthreads();
    for (int i = threadIdx.x; i < (rows + 31) / 32; i += kSumThreads) present[i] = 0u;
    __syncthreads();
#pragma unroll 16
    for (int i = threadIdx.x; i < n; i += kSumThreads) {
      const int r = __ldg(z.ids + i) - lo;
      if (r >= 0 && r < rows) atomicOr(present + (r >> 5), 1u << (r & 31));
    }
    __syncthreads();
    auto absent = [&](int r) { return (present[r >> 5] >> (r & 31) & 1) == 0; };
    const int64_t row_bytes = (int64_t)hidden * sizeof(O);
    if (out_stride == hidden && row_bytes >= 16 && row_bytes < 1024) {
      // short rows next to each other: windows of all of them, over at most two rows each
      // (a warp a row took 48 us for 128566 rows of 94 bf16, 24 MB)
      const uintptr_t start = reinterpret_cast<uintptr_t>(out + (int64_t)lo * out_stride);
      const uintptr_t end = start + (uintptr_t)(rows * row_bytes);
      for (uintptr_t w = (start & ~(uintptr_t)15) + 16 * (uintptr_t)threadIdx.x; w < end; w += 16 * kSumThreads) {
        const uint32_t at = w < start ? 0u : (uint32_t)(w - start), past = (uint32_t)((w + 15 < end ? w + 15 : end - 1) - start);
        const int r0 = (int)(at / (uint32_t)row_bytes), r1 = (int)(past / (uint32_t)row_bytes);
        const bool a0 = absent(r0), a1 = absent(r1);
        const uint4 zero = make_uint4(0, 0, 0, 0);
        if (a0 && a1 && w >= start && w + 16 <= end) *reinterpret_cast<uint4 *>(w) = zero;
        else if (a0 || a1) {
          const uintptr_t border = start + (uintptr_t)(r1 * row_bytes);
          write_edge<O>(zero, w, a0 ? start : border, a1 ? end : border);
        }
      }
      continue;
    }
    for (int r = threadIdx.x >> 5; r < rows; r += kSumThreads / 32) {
      if (!absent(r)) continue;
      // whole windows of the row, its ends by element (by element alone 3.2 TB/s of bf16)
      const uintptr_t start = reinterpret_cast<uintptr_t>(out + (int64_t)(lo + r) * out_stride);
      const uintptr_t end = start + (uintptr_t)hidden * sizeof(O);
      const uint4 zero = make_uint4(0, 0, 0, 0);
      for (uintptr_t w = (start & ~(uintptr_t)15) + 16 * (uintptr_t)lane; w < end; w += 512) {
        if (w >= start && w + 16 <= end) *reinterpret_cast<uint4 *>(w) = zero;
        else write_edge<O>(zero, w, start, end);
      }
    }
  }
}

struct SumArgs {
  const uint2 *items;  // sorted
  int n, piece, vocab, hidden;
  int64_t stride, out_stride;
  ZeroArgs zero;  // by the first CTAs of a kernel
  float scale;
  bool accumulate;
  float *partial;  // [pieces][2][hidden]: of the run from the piece before, of the run into the next
};

// acc (fp32, as the columns of RowPart<., V, 8>) scaled, or added, into a row.
template <typename O, int V>
__device__ __forceinline__ void write_row(const float (&acc)[8], const SumArgs &a, O *row, int t,
                                          int threads, int width) {
  RowPart<O, V, 8> o;
  if (a.accumulate) {
    o.template load<true>(row, t, threads, width);
#pragma unroll
    for (int e = 0; e < 8; e += 2)
      o.set2(e, fmaf(acc[e], a.scale, o.get(e)), fmaf(acc[e + 1], a.scale, o.get(e + 1)));
  } else {
#pragma unroll
    for (int e = 0; e < 8; e += 2) o.set2(e, acc[e] * a.scale, acc[e + 1] * a.scale);
  }
  o.store(row, t, threads, width);
}

// A group of TPR threads sums a piece: runs inside it go to the table, its first
// and last run to `partial` where they cross its border.
template <typename T, typename O, int V, int TPR>
__global__ void __launch_bounds__(kSumThreads)
    embed_sum_kernel(const T *__restrict__ grad, SumArgs a, O *out) {
  constexpr int kLoads = 4;
  const int t = threadIdx.x % TPR;
  if ((int)blockIdx.x < a.zero.ctas) {
    pdl_launch_dependents();
    if (blockIdx.y == 0) write_zeros(a.zero, a.n, a.hidden, out, a.out_stride);
    return;
  }
  const int piece = ((int)blockIdx.x - a.zero.ctas) * (kSumThreads / TPR) + threadIdx.x / TPR;
  const int c0 = blockIdx.y * TPR * 8, width = a.hidden - c0;
  pdl_wait_primary();
  pdl_launch_dependents();
  if ((int64_t)piece * a.piece >= a.n) return;
  const int s = piece * a.piece, end = min(s + a.piece, a.n);
  const uint32_t before = s > 0 ? __ldcg(&a.items[s - 1].x) : ~0u;
  const uint32_t after = end < a.n ? __ldcg(&a.items[end].x) : ~0u;
  float acc[8];
  uint32_t run = ~0u;
  int start = s;
  auto flush = [&](int stop) {
    if (run >= (uint32_t)a.vocab) return;
    if ((start == s && before == run) || (stop == end && after == run)) {
      RowPart<float, V, 8> p;
#pragma unroll
      for (int e = 0; e < 8; e += 2) p.set2(e, acc[e], acc[e + 1]);
      // (rows of `partial` are as far from 16 bytes as a row's length: by elements then)
      float *row = a.partial + ((int64_t)piece * 2 + (start == s ? 0 : 1)) * a.hidden + c0;
      p.store(row, t, TPR, width);
    } else {
      write_row<O, V>(acc, a, out + (int64_t)run * a.out_stride + c0, t, TPR, width);
    }
  };
  for (int i = s; i < end; i += kLoads) {
    uint2 it[kLoads];
    RowPart<T, V, 8> p[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) it[j] = i + j < end ? __ldcg(a.items + i + j) : make_uint2(~0u, 0);
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      if (it[j].x < (uint32_t)a.vocab) p[j].load(grad + (int64_t)it[j].y * a.stride + c0, t, TPR, width);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      if (it[j].x >= (uint32_t)a.vocab) continue;  // padding, sorted last
      if (it[j].x != run) {
        flush(i + j);
        run = it[j].x;
        start = i + j;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += p[j].get(e);
    }
  }
  // (where padding follows the last run, `after` is its key and not the run's)
  flush(end);
}

// A run that crosses pieces: the group of the piece where it begins adds the
// pieces' sums in order.
template <typename O, int V, int TPR>
__global__ void __launch_bounds__(kSumThreads, 3) embed_join_kernel(SumArgs a, O *out) {
  const int t = threadIdx.x % TPR, lane = threadIdx.x & 31;
  if ((int)blockIdx.x < a.zero.ctas) {
    pdl_launch_dependents();
    if (blockIdx.y == 0) write_zeros(a.zero, a.n, a.hidden, out, a.out_stride);
    return;
  }
  const int piece = ((int)blockIdx.x - a.zero.ctas) * (kSumThreads / TPR) + threadIdx.x / TPR;
  const int c0 = blockIdx.y * TPR * 8, width = a.hidden - c0;
  pdl_wait_primary();
  pdl_launch_dependents();
  if ((int64_t)(piece + 1) * a.piece >= a.n) return;
  // (the keys around the piece and where the next 32 begin at once: their latency, with the
  // sums', is what a join of two pieces takes)
  const int s = piece * a.piece, end = s + a.piece;
  const int64_t starts = (int64_t)(piece + 1 + lane) * a.piece;
  const uint32_t run = __ldcg(&a.items[end - 1].x), first = __ldcg(&a.items[s].x);
  const uint32_t before = s > 0 ? __ldcg(&a.items[s - 1].x) : ~0u;
  uint32_t in = __ballot_sync(0xFFFFFFFFu, starts < a.n && __ldcg(&a.items[starts < a.n ? starts : s].x) == run);
  if (run >= (uint32_t)a.vocab || (in & 1u) == 0) return;
  const bool whole = first == run;
  if (whole && before == run) return;  // begins before
  // pieces that it reaches: those whose first position still is the run's
  int last = piece;
  for (;;) {
    const int n = in == 0xFFFFFFFFu ? 32 : __ffs(~in) - 1;
    last += n;
    if (n < 32) break;
    const int64_t at = (int64_t)(last + 1 + lane) * a.piece;
    in = __ballot_sync(0xFFFFFFFFu, at < a.n && __ldcg(&a.items[at].x) == run);
  }
  float acc[8];
  RowPart<float, V, 8> p;
  p.template load<true>(a.partial + ((int64_t)piece * 2 + (whole ? 0 : 1)) * a.hidden + c0, t, TPR, width);
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = p.get(e);
  // what it takes is the loads' latency: several at a time, with room for three CTAs on an SM
  // (28042 ids of 8232 tokens, 1088 fp32: all of the gradient 59 us; 12 at a time and two CTAs
  // 68, but 32768 times the same token, 1024 bf16, 100 in place of 123), without conditions (columns
  // past the row's end read its last ones and are not stored; rows past the last
  // piece read that one and are not added)
  constexpr int kLoads = 6;
  const float *row = a.partial + c0;
  for (int k = piece + 1; k <= last; k += kLoads) {
    float q[kLoads][8];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const float *from = row + (int64_t)min(k + j, last) * 2 * a.hidden;
#pragma unroll
      for (int e = 0; e < 8; e += V) {
        const float *at = from + min(RowPart<float, V, 8>::column(e, t, TPR), width - V);
        if constexpr (V == 1) {
          q[j][e] = __ldcg(at);
        } else {
#pragma unroll
          for (int i = 0; i < V; i += 4) {
            const float4 v = __ldcg(reinterpret_cast<const float4 *>(at + i));
            q[j][e + i] = v.x; q[j][e + i + 1] = v.y; q[j][e + i + 2] = v.z; q[j][e + i + 3] = v.w;
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += k + j <= last ? q[j][e] : 0.0f;
  }
  write_row<O, V>(acc, a, out + (int64_t)run * a.out_stride + c0, t, TPR, width);
}

int piece_rows(int rows) {
  int p = kLeastPiece;
  while (p < kMostPiece && (int64_t)p * kSms * 8 < rows) p *= 2;
  return p;
}

size_t items_bytes(int rows) { return align_up((size_t)rows * sizeof(uint2), 256); }

// The tokens whose zeros the joining kernel writes, the last of the table: a few
// microseconds' worth, as long as its joins wait for their loads, and none where many ids
// would have to be read for them.
int zeros_of_joins(int rows, int pieces, int hidden, int vocab, int element_bytes) {
  if (pieces < 2 || rows > 65536) return 0;
  const int64_t most = ((int64_t)40 << 20) / ((int64_t)hidden * element_bytes);
  return (int)(most < vocab / 5 ? most : vocab / 5);
}

template <typename T, typename O, int V, int TPR>
cudaError_t sum_pieces(const T *grad, SumArgs a, O *out, cudaStream_t stream) {
  const int pieces = (a.n + a.piece - 1) / a.piece, groups = kSumThreads / TPR;
  const unsigned blocks = (unsigned)((pieces + groups - 1) / groups), strips = (unsigned)((a.hidden + TPR * 8 - 1) / (TPR * 8));
  const bool zero = a.zero.ctas > 0;
  const int later = zero ? zeros_of_joins(a.n, pieces, a.hidden, a.vocab, sizeof(O)) : 0;
  a.zero.to = a.vocab - later;
  // (without rows the sort has not been launched: nothing to start beside)
  cudaError_t err = launch_chained(embed_sum_kernel<T, O, V, TPR>, dim3(blocks + a.zero.ctas, strips),
                                   dim3(kSumThreads), 0, stream, 1, a.n > 0, grad, a, out);
  if (err != cudaSuccess || pieces < 2) return err;
  a.zero.from = a.zero.to;
  a.zero.to = a.vocab;
  if (!later) a.zero.ctas = 0;
  return launch_chained(embed_join_kernel<O, V, TPR>, dim3(blocks + a.zero.ctas, strips), dim3(kSumThreads), 0,
                        stream, 1, true, a, out);
}

template <typename T, typename O, int V>
cudaError_t sum_rows(const T *grad, const SumArgs &a, O *out, cudaStream_t stream) {
  return a.hidden <= 256    ? sum_pieces<T, O, V, 32>(grad, a, out, stream)
         : a.hidden <= 512  ? sum_pieces<T, O, V, 64>(grad, a, out, stream)
         : a.hidden <= 1024 ? sum_pieces<T, O, V, 128>(grad, a, out, stream)
                            : sum_pieces<T, O, V, 256>(grad, a, out, stream);
}

cudaError_t sort_rows(const SortArgs &s, cudaStream_t stream) {
  static std::atomic<uint64_t> ready{0};
  const cudaError_t err = allow_shared(ready, (const void *)embed_sort_kernel, (int)sizeof(SortShared));
  if (err != cudaSuccess) return err;
  // one CTA while its lanes hold all items
  const int ctas = s.n <= kSortThreads * kHeldItems ? 1 : kSortCtas;
  return launch_chained(embed_sort_kernel, dim3(ctas), dim3(kSortThreads), sizeof(SortShared), stream, ctas, false, s);
}

template <typename T, typename O>
cudaError_t embed_grad(const T *grad, int rows, int hidden, int64_t stride, const int32_t *ids,
                       float scale, O *out, int vocab, int64_t out_stride, bool accumulate,
                       void *workspace, cudaStream_t stream) {
  char *w = static_cast<char *>(workspace);
  const SortArgs s = {ids, rows, vocab, reinterpret_cast<uint2 *>(w),
                      reinterpret_cast<uint2 *>(w + items_bytes(rows))};
  const SumArgs a = {s.a, rows, piece_rows(rows), vocab, hidden, stride, out_stride,
                     {ids, accumulate ? 0 : kZeroCtas, 0, vocab}, scale, accumulate,
                     reinterpret_cast<float *>(w + 2 * items_bytes(rows))};
  const void *base[1] = {out};
  const int64_t strides[1] = {out_stride};
  const int vo = row_vector(sizeof(O), hidden, 1, base, strides);
  if (rows > 0) {
    const cudaError_t err = sort_rows(s, stream);
    if (err != cudaSuccess) return err;
  }
  // one access for the gradient's rows, the table's and the sums': whole 16 bytes
  // of the gradient's type, else element by element
  const void *gbase[1] = {grad};
  const int64_t gstrides[1] = {stride};
  const int vg = row_vector(sizeof(T), hidden, 1, gbase, gstrides);
  if (vg * sizeof(T) == 16 && vo * sizeof(O) == 16)
    return sum_rows<T, O, 16 / sizeof(T)>(grad, a, out, stream);
  return sum_rows<T, O, 1>(grad, a, out, stream);
}

}  // namespace

cudaError_t launch_embed(const void *table, int dtype, int vocab, int hidden, int64_t stride,
                         const int32_t *ids, int rows, float scale, void *out, int64_t out_stride,
                         cudaStream_t stream) {
  const void *base[2] = {table, out};
  const int64_t strides[2] = {stride, out_stride};
  const int v = row_vector(dtype == SLIMWISE_DTYPE_BF16 ? 2 : 4, hidden, 2, base, strides);
  auto go = [&](auto kernel, auto *tab, auto *o, int strip) {
    const int64_t warps = (int64_t)rows * ((hidden + strip - 1) / strip);
    const int64_t ctas = (warps + kLookupThreads / 32 - 1) / (kLookupThreads / 32);
    const int64_t most = (int64_t)kSms * 64;
    kernel<<<(unsigned)(ctas < most ? ctas : most), kLookupThreads, 0, stream>>>(
        tab, vocab, hidden, stride, ids, rows, scale, o, out_stride);
    return cudaGetLastError();
  };
  if (dtype == SLIMWISE_DTYPE_BF16) {
    const auto *tab = static_cast<const __nv_bfloat16 *>(table);
    auto *o = static_cast<__nv_bfloat16 *>(out);
    if (v == 8) return go(embed_kernel<__nv_bfloat16, 8>, tab, o, 32 * 8 * kLookupLoads);
    if (v == 2) return go(embed_kernel<__nv_bfloat16, 2>, tab, o, 32 * 2 * kLookupLoads);
    return go(embed_kernel<__nv_bfloat16, 1>, tab, o, 32 * 2 * kLookupLoads);
  }
  const auto *tab = static_cast<const float *>(table);
  auto *o = static_cast<float *>(out);
  if (v == 4) return go(embed_kernel<float, 4>, tab, o, 32 * 4 * kLookupLoads);
  return go(embed_kernel<float, 1>, tab, o, 32 * kLookupLoads);
}

size_t embed_grad_workspace(int rows, int hidden) {
  const size_t piece = (size_t)piece_rows(rows), pieces = ((size_t)rows + piece - 1) / piece;
  return 2 * items_bytes(rows) + pieces * 2 * hidden * sizeof(float) + 256;
}

cudaError_t launch_embed_grad(const void *grad, int dtype, int rows, int hidden, int64_t stride,
                              const int32_t *ids, float scale, void *out, int out_dtype, int vocab,
                              int64_t out_stride, bool accumulate, void *workspace,
                              cudaStream_t stream) {
  auto go = [&](auto *g, auto *o) {
    return embed_grad(g, rows, hidden, stride, ids, scale, o, vocab, out_stride, accumulate, workspace,
                      stream);
  };
  const auto *gb = static_cast<const __nv_bfloat16 *>(grad);
  const auto *gf = static_cast<const float *>(grad);
  auto *ob = static_cast<__nv_bfloat16 *>(out);
  auto *of = static_cast<float *>(out);
  if (dtype == SLIMWISE_DTYPE_BF16) return out_dtype == SLIMWISE_DTYPE_BF16 ? go(gb, ob) : go(gb, of);
  return out_dtype == SLIMWISE_DTYPE_BF16 ? go(gf, ob) : go(gf, of);
}

}  // namespace slimwise
