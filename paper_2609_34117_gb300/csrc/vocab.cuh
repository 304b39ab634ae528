// vocab.cuh -- what the operators over rows of vocabulary logits share: the
// 16-byte windows a row is read in, order-preserving keys, block reductions,
// and the streaming pass that finds a row's largest elements and the sum of
// its exponentials in one read.
//
// A row of V elements starts anywhere (odd vocabularies make odd rows), so it
// is seen as the 16-byte windows that cover it: window w holds elements
// w E - mis .. + E - 1, E = 16 / sizeof(T), mis = the row's offset from a
// 16-byte boundary.  Only the first and the last window can be partial; those
// are read element by element, with -inf outside the row, which neither a
// maximum nor a sum of exponentials sees.
#pragma once

#include <cooperative_groups.h>
#include <float.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"

namespace slimwise {

constexpr int kVocabMax = 393216;   // longest row (the loss keeps a row in a cluster's shared memories)
constexpr int kTopMax = 256;        // longest list of top logits
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// Stands in for -inf as the reference of a sum of exponentials, so that
// z - reference of a z of -inf is -inf.
constexpr float kFloorRef = -FLT_MAX;

// Launches `clusters` clusters of C CTAs.  smem_max: the kernel's shared-memory
// attribute, one value per kernel; smem: this launch's.
template <typename K, typename... A>
inline cudaError_t launch_clusters(K kernel, int clusters, int C, int threads, size_t smem,
                                   size_t smem_max, cudaStream_t stream, A... args) {
  cudaError_t err = cudaFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                         cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)smem_max);
  if (err != cudaSuccess) return err;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)clusters * (unsigned)C);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

cudaError_t launch_top_logits(const void *logits, int dtype, int rows, int vocab, int64_t stride,
                              int k, float temperature, int32_t *ids, float *logp, float *log_rest,
                              cudaStream_t stream);
cudaError_t launch_sample(const void *logits, int dtype, int rows, int vocab, int64_t stride,
                          const float *temperature, const int32_t *top_k, const float *top_p,
                          const float *min_p, const float *uniform, int32_t *tokens,
                          float *logprob, cudaStream_t stream);
cudaError_t launch_distill_loss(const void *logits, int dtype, int rows, int vocab, int64_t stride,
                                const int32_t *labels, const int32_t *top_ids,
                                const float *top_logp, const float *log_rest, int k, float alpha,
                                float temperature, const float *row_weight, float *row_loss,
                                float *loss, void *grad, int64_t grad_stride, cudaStream_t stream);

// How a scan is launched: CTAs of a cluster (a row is split over them), and
// clusters, each of which takes every clusters-th row.
struct ScanGrid {
  int C, clusters;
};
ScanGrid scan_grid(int rows, int vocab, int element_bytes, int ctas_per_sm);

#if defined(__CUDACC__)
namespace cg = cooperative_groups;

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Order-preserving map of a number to 1 .. 2^32 - 1 (-0 folded onto +0).
__device__ __forceinline__ uint32_t ordered(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return (b >> 31) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
  return __uint_as_float((o >> 31) ? (o & 0x7FFFFFFFu) : ~o);
}
// A key of its own for each element (or window): larger value first, then the
// lower index.  0 is no key.
__device__ __forceinline__ uint64_t make_key(float z, uint32_t idx) {
  return ((uint64_t)ordered(z) << 32) | (0xFFFFFFFFu - idx);
}
__device__ __forceinline__ float key_value(uint64_t k) { return unordered((uint32_t)(k >> 32)); }
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xFFFFFFFFu - (uint32_t)k; }

// Rows as windows ------------------------------------------------------------
template <typename T>
struct Row {
  static constexpr int E = 16 / (int)sizeof(T);
  const T *p;      // first element
  const uint4 *w;  // window 0 (the 16-byte boundary at or before p)
  int vocab, mis, windows;
  __device__ __forceinline__ Row(const T *row, int V) : p(row), vocab(V) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(row);
    mis = (int)((a & 15) / sizeof(T));
    w = reinterpret_cast<const uint4 *>(a & ~(uintptr_t)15);
    windows = (mis + V + E - 1) / E;
  }
  __device__ __forceinline__ bool whole(int i) const {
    return i * E >= mis && (i + 1) * E <= mis + vocab;
  }
};

__device__ __forceinline__ uint32_t neg_inf_bits(const __nv_bfloat16 *) { return 0xFF80FF80u; }
__device__ __forceinline__ uint32_t neg_inf_bits(const float *) { return 0xFF800000u; }

// Window i of the row, -inf outside the row.
template <typename T>
__device__ __forceinline__ uint4 load_window(const Row<T> &r, int i) {
  if (r.whole(i)) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(r.w + i));
    return v;
  }
  constexpr int E = Row<T>::E;
  uint32_t u[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) u[q] = neg_inf_bits(r.p);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int id = i * E - r.mis + e;
    if (id >= 0 && id < r.vocab) {
      if constexpr (sizeof(T) == 4) {
        u[e] = reinterpret_cast<const uint32_t *>(r.p)[id];
      } else {
        const uint32_t b = reinterpret_cast<const uint16_t *>(r.p)[id];
        u[e >> 1] = (e & 1) ? ((u[e >> 1] & 0xFFFFu) | (b << 16)) : ((u[e >> 1] & 0xFFFF0000u) | b);
      }
    }
  }
  return make_uint4(u[0], u[1], u[2], u[3]);
}

template <typename T>
__device__ __forceinline__ void unpack(const uint4 &v, float (&f)[16 / sizeof(T)]) {
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (sizeof(T) == 4) {
      f[q] = __uint_as_float(u[q]);
    } else {
      f[2 * q] = __uint_as_float(u[q] << 16);
      f[2 * q + 1] = __uint_as_float(u[q] & 0xFFFF0000u);
    }
  }
}

// Largest element of a window (NaN only if all are).
template <typename T>
__device__ __forceinline__ float window_max(const uint4 &v) {
  if constexpr (sizeof(T) == 4) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)),
                 fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  } else {
    uint32_t m, n;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(v.x), "r"(v.y));
    asm("max.bf16x2 %0, %1, %2;" : "=r"(n) : "r"(v.z), "r"(v.w));
    asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(m), "r"(n));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
  }
}

// Bulk copy of whole windows into shared memory, counted on an mbarrier.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
      "l"(src), "r"(bytes), "r"(bar)
      : "memory");
}
// Waits for a copy; false after a second without it.
__device__ __forceinline__ bool wait_copy(uint32_t bar, uint32_t parity) {
#pragma unroll 1
  for (int i = 0; i < 256; ++i)
    if (mbar_try_wait(bar, parity)) return true;
  return mbar_wait_timeout(bar, parity, kDefaultWaitLimitNs);
}

// Two floats in one register pair: one instruction works on both.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(a), "f"(b));
  return p;
}
__device__ __forceinline__ void split(uint64_t p, float &a, float &b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p));
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// 2^((z - ref) c), the difference first: it is exact where it matters, and no
// product of a masked logit overflows.
__device__ __forceinline__ float exp_from(float z, float ref, float c) { return ex2((z - ref) * c); }
// The same of a pair.
__device__ __forceinline__ uint64_t exp2_pair(uint64_t z, uint64_t minus_ref, uint64_t cc) {
  float a, b;
  split(mul2(add2(z, minus_ref), cc), a, b);
  return pair(ex2(a), ex2(b));
}

// The window's elements as pairs, in order.
template <typename T>
__device__ __forceinline__ void unpack_pairs(const uint4 &v, uint64_t (&p)[8 / sizeof(T)]) {
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
  if constexpr (sizeof(T) == 4) {
    p[0] = pair(__uint_as_float(u[0]), __uint_as_float(u[1]));
    p[1] = pair(__uint_as_float(u[2]), __uint_as_float(u[3]));
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      p[q] = pair(__uint_as_float(u[q] << 16), __uint_as_float(u[q] & 0xFFFF0000u));
  }
}

// Sum over the window of 2^((z - ref) c).
template <typename T>
__device__ __forceinline__ float window_sum(const uint4 &v, float c, float ref) {
  constexpr int P = 8 / (int)sizeof(T);
  uint64_t p[P];
  unpack_pairs<T>(v, p);
  const uint64_t mr = pair(-ref, -ref), cc = pair(c, c);
#pragma unroll
  for (int q = 0; q < P; ++q) p[q] = exp2_pair(p[q], mr, cc);
#pragma unroll
  for (int d = 1; d < P; d *= 2)
#pragma unroll
    for (int q = 0; q < P; q += 2 * d) p[q] = add2(p[q], p[q + d]);
  float a, b;
  split(p[0], a, b);
  return a + b;
}

// Block reductions over NT threads; every thread gets the result.  `buf` has
// room for NT / 32 values and is free again after the call.
template <int NT, typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, V *buf, F f) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) v = f(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = buf[0];
#pragma unroll
  for (int w = 1; w < NT / 32; ++w) v = f(v, buf[w]);
  __syncthreads();
  return v;
}
struct OpAdd {
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};
struct OpMax {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// Scanning rows for their largest elements ---------------------------------------
// A row is read once, and the scan leaves (a) every element that is not below a
// threshold under which fewer than K of the row's elements cannot lie, and (b)
// the sum of the exponentials of all others.
//
// The threshold: each thread keeps the largest element of two groups of
// windows.  If K groups reach a value, K elements do, so the K-th largest group
// maximum bounds the K-th largest element from below, and with many more groups
// than K it is near it, however long the row: of 512 groups, about
// -512 ln(1 - K / 512) elements lie above it (68 for K = 64).  It is found by
// bisection with block-wide counts, after the 1st, 2nd, 4th, ... step, so that
// each doubling of what was read lists that many windows again and no more.  A
// window whose maximum reaches the threshold is listed with its sum; any other
// only adds its sum to the thread's.
//
// The K largest elements of a row lie in the K windows of largest maximum (ties:
// lower index), since each of those holds an element that goes before every
// element of the others.  So a list that fills (many equal values, or rows in
// rising order) is cut to its K best windows by a radix selection, and nothing
// that matters is lost.
//
// Sums are relative to the threshold, not to the maximum: what lies below the
// list keeps its precision however far the list rises above it.  Which thread
// adds what never depends on timing, so that results are the same on every run.
//
// Each warp streams its windows through a ring of its own with bulk copies; a
// stage is copied again as soon as its windows are in registers, and the copies
// of the next row are under way while a row is finished.
constexpr int kScanThreads = 256;
constexpr int kScanWarps = kScanThreads / 32;
constexpr int kScanUnroll = 4;                          // windows of a lane in a step
constexpr int kWarpStep = 32 * kScanUnroll;             // windows of a warp in a step
constexpr int kScanStep = kScanThreads * kScanUnroll;   // windows of a CTA in a step
constexpr int kScanStages = 2;
constexpr int kListWarp = 192;                          // listed windows of a warp
constexpr int kListSlots = kScanWarps * kListWarp / kScanThreads;  // of a thread
constexpr int kClusterMax = 8;
static_assert(kTopMax <= kScanThreads, "a thread for each kept window and candidate");
static_assert(kTopMax / kScanWarps + kWarpStep <= kListWarp, "room for a step after a cut");

// Candidates that a CTA passes on: the K best and others, if there are no more
// than this (else the K best alone).
__host__ __device__ inline int candidate_cap(int K) {
  return K >= 128 ? kTopMax : K <= 32 ? 64 : 2 * K;
}

struct ScanShared {
  uint4 ring[kScanWarps][kScanStages][kWarpStep];
  uint64_t key[kScanWarps][kListWarp];
  float sum[kScanWarps][kListWarp];  // of 2^((z - the window's maximum) c)
  uint64_t cand[kTopMax];
  uint64_t bar[kScanWarps][kScanStages];
  uint64_t red64[kScanWarps];
  uint32_t hist[256];
  float by_rank[kTopMax];
  float redf[kScanWarps];
  uint32_t redu[2][kScanWarps];
  int count[kScanWarps];
  int sel_digit, sel_above, sel_bin;
  int late;                                  // a wait for a copy gave up
  float part_sum[kClusterMax], part_thr[kClusterMax];  // at a row's leader: each CTA's
  int part_exact[kClusterMax];
  // then, in clusters: uint64_t [cluster][cap], each CTA's candidates at a row's leader
};

// The bits of v from bit `from` (up to 64) up.
__device__ __forceinline__ uint64_t high_bits(uint64_t v, int from) {
  return from >= 64 ? 0 : v >> from << from;
}

// Threshold such that exactly K of the keys in the block's registers (0: none)
// are at least it; more than K are not 0.  A radix selection from the highest
// bit in which they differ, 8 bits a pass, that ends when a whole bin is taken.
template <int N>
__device__ __forceinline__ uint64_t select_kth(const uint64_t (&k)[N], int K, ScanShared &sh) {
  const int tid = threadIdx.x;
  uint32_t hi_or = 0, hi_and = 0xFFFFFFFFu;
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (k[j]) {
      hi_or |= (uint32_t)(k[j] >> 32);
      hi_and &= (uint32_t)(k[j] >> 32);
    }
  hi_or = __reduce_or_sync(0xFFFFFFFFu, hi_or);
  hi_and = __reduce_and_sync(0xFFFFFFFFu, hi_and);
  __syncthreads();
  if ((tid & 31) == 0) {
    sh.redu[0][tid >> 5] = hi_or;
    sh.redu[1][tid >> 5] = hi_and;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kScanWarps; ++w) {
    hi_or |= sh.redu[0][w];
    hi_and &= sh.redu[1][w];
  }
  const uint32_t diff = hi_or ^ hi_and;
  int shift = diff ? (32 + 31 - __clz((int)diff)) - 7 : 24;
  int known = shift + 8;  // bits from here up are settled: the prefix's
  uint64_t prefix = high_bits((uint64_t)hi_and << 32, known);
  int need = K;
  while (true) {
    sh.hist[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (k[j] && high_bits(k[j], known) == prefix)
        atomicAdd(&sh.hist[(uint32_t)(k[j] >> shift) & 255u], 1u);
    __syncthreads();
    if (tid < 32) {
      // lane l takes bins 8 l .. 8 l + 7; keys in higher bins come first
      int c[8], mine = 0;
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        c[b] = (int)sh.hist[8 * tid + b];
        mine += c[b];
      }
      int incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_down_sync(0xFFFFFFFFu, incl, o);
        if (tid + o < 32) incl += v;
      }
      int above = incl - mine;
      if (above < need && need <= incl) {
#pragma unroll
        for (int b = 7; b >= 0; --b) {
          if (above < need && need <= above + c[b]) {
            sh.sel_digit = 8 * tid + b;
            sh.sel_above = above;
            sh.sel_bin = c[b];
          }
          above += c[b];
        }
      }
    }
    __syncthreads();
    need -= sh.sel_above;
    prefix |= (uint64_t)sh.sel_digit << shift;
    const bool done = sh.sel_bin == need || shift == 0;
    __syncthreads();
    if (done) return prefix;
    known = shift;
    shift = max(shift - 8, 0);
  }
}

// Exclusive prefix sum of v over the block; `total` the sum.
__device__ __forceinline__ int block_prefix(int v, int &total, ScanShared &sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += u;
  }
  if (lane == 31) sh.redu[0][warp] = (uint32_t)incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kScanWarps; ++w) {
    if (w < warp) before += (int)sh.redu[0][w];
    total += (int)sh.redu[0][w];
  }
  __syncthreads();
  return before + incl - v;
}

template <typename T>
struct Scan {
  static constexpr int E = Row<T>::E;
  ScanShared &sh;
  uint64_t *recv;  // behind sh
  int recv_cap;    // candidates of a CTA that recv has room for
  const T *logits;
  int64_t stride;
  int vocab, rows;
  int C, rank, clusters;        // CTAs of a cluster, this CTA's place, clusters of the grid
  int lane, warp;
  // the copies under way: step next_k of row next_t
  int next_t, next_k;
  uint32_t issued, used;        // stages copied, and read
  // the row at hand
  int lo, hi, K;
  float c, thr;                 // scale of the exponents (log2 e / temperature); threshold
  float list_thr;               // maximum at which a window is listed: thr, or just above it
  float ref, s, lost;           // s, with its low part: sum of 2^((z - ref) c) of what is not listed
  bool exact;                   // the K best alone are known to be complete
  bool dead;                    // a copy did not arrive: this warp waits for none any more
  float top0, top1;             // maxima of this thread's groups
  int listed;                   // windows in this warp's list

  __device__ __forceinline__ Scan(ScanShared &shared, int cap, const T *z, int64_t st, int V, int n)
      : sh(shared), recv(reinterpret_cast<uint64_t *>(&shared + 1)), recv_cap(cap), logits(z),
        stride(st), vocab(V), rows(n), dead(false) {
    cg::cluster_group cluster = cg::this_cluster();
    C = (int)cluster.num_blocks();
    rank = (int)cluster.block_rank();
    clusters = (int)gridDim.x / C;
    lane = threadIdx.x & 31;
    warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
      for (int w = 0; w < kScanWarps; ++w)
        for (int i = 0; i < kScanStages; ++i) mbar_init(smem_u32(&sh.bar[w][i]), 1);
      mbar_fence_init();
      sh.late = 0;
    }
    __syncthreads();
    next_t = (int)(blockIdx.x / C);
    next_k = 0;
    issued = used = 0;
    for (int i = 0; i < kScanStages; ++i) issue();
    if (C > 1) cluster_arrive();  // every CTA runs before another writes to its shared memory
    waited = C == 1;
  }
  __device__ __forceinline__ Row<T> row_of(int t) const {
    return Row<T>(logits + (int64_t)t * stride, vocab);
  }
  __device__ __forceinline__ void slice(const Row<T> &row, int &a, int &b) const {
    const int per = (row.windows + C - 1) / C;
    a = min(rank * per, row.windows);
    b = min(a + per, row.windows);
  }

  // Starts the copy of this warp's windows of the next step; the row's partial
  // windows at its ends are left out.
  __device__ __forceinline__ void issue() {
    if (next_t >= rows || dead) return;
    const Row<T> row = row_of(next_t);
    int a, b;
    slice(row, a, b);
    const int stage = (int)(issued % kScanStages);
    const int i0 = a + next_k * kScanStep + warp * kWarpStep;
    int first = i0, end = min(i0 + kWarpStep, b);
    if (first == 0 && !row.whole(0)) ++first;
    if (end == row.windows && end > first && !row.whole(end - 1)) --end;
    const uint32_t bar = smem_u32(&sh.bar[warp][stage]);
    __syncwarp();
    if (elect_one()) {
      const uint32_t bytes = end > first ? (uint32_t)(end - first) * 16 : 0;
      mbar_arrive_expect_tx(bar, bytes);
      if (bytes) bulk_load(smem_u32(&sh.ring[warp][stage][first - i0]), row.w + first, bytes, bar);
    }
    ++issued;
    if (a + (++next_k) * kScanStep >= b) {
      next_k = 0;
      next_t += clusters;
    }
  }
  // Waits for the oldest copy; a wait that gives up marks the CTA's results.
  __device__ __forceinline__ int wait() {
    const int stage = (int)(used % kScanStages);
    if (!dead) {
      const bool ok = wait_copy(smem_u32(&sh.bar[warp][stage]), (used / kScanStages) & 1);
      if (!__all_sync(0xFFFFFFFFu, ok)) {
        dead = true;
        sh.late = 1;
      } else {
        ++used;
      }
    }
    return stage;
  }

  __device__ __forceinline__ int groups_at(float x) const {
    return __syncthreads_count(top0 >= x) + __syncthreads_count(top1 >= x);
  }
  // Raises the threshold to what the groups show, and drops the listed windows
  // below it.
  __device__ __forceinline__ void refresh() {
    // bounds to search between: the groups' largest, and the threshold at hand
    // or (the first time) the groups' least
    const float least = fminf(top0 > -INFINITY ? top0 : INFINITY, top1 > -INFINITY ? top1 : INFINITY);
    const uint32_t h = __reduce_max_sync(0xFFFFFFFFu, ordered(fmaxf(top0, top1)));
    const uint32_t l = __reduce_min_sync(0xFFFFFFFFu, ordered(least));
    if (lane == 0) {
      sh.redu[0][warp] = h;
      sh.redu[1][warp] = l;
    }
    __syncthreads();
    uint32_t high = 0, low = 0xFFFFFFFFu;
#pragma unroll
    for (int w = 0; w < kScanWarps; ++w) {
      high = max(high, sh.redu[0][w]);
      low = min(low, sh.redu[1][w]);
    }
    bool known = true;  // K groups reach `low`
    if (thr > -INFINITY) low = ordered(thr);
    else known = low <= high && groups_at(unordered(low)) >= K;
    if (known) {
      while (high - low > 1) {
        const uint32_t mid = low + (high - low) / 2;
        const int n = groups_at(unordered(mid));
        if (n >= K) {
          low = mid;
          if (n <= K + K / 8) break;
        } else {
          high = mid;
        }
      }
      if (unordered(low) > thr) {
        raise(unordered(low));
        list_thr = thr;
      }
    }
    __syncthreads();
    int out = 0;
    for (int base = 0; base < listed; base += 32) {
      const int i = base + lane;
      uint64_t k = 0;
      float ws = 0.0f;
      if (i < listed) {
        k = sh.key[warp][i];
        ws = sh.sum[warp][i];
      }
      const bool keep = k && key_value(k) >= thr;
      const uint32_t mask = __ballot_sync(0xFFFFFFFFu, keep);
      if (keep) {
        const int at = out + __popc(mask & ((1u << lane) - 1u));
        sh.key[warp][at] = k;
        sh.sum[warp][at] = ws;
      } else if (k) {
        drop(k, ws);
      }
      out += __popc(mask);
      __syncwarp();
    }
    listed = out;
  }
  __device__ __forceinline__ void raise(float low) {
    thr = low;
    const float r = fmaxf(thr, kFloorRef), f = exp_from(ref, r, c);
    s *= f;
    lost *= f;
    ref = r;
  }
  __device__ __forceinline__ void drop(uint64_t k, float ws) {
    s += ws * exp_from(fmaxf(key_value(k), kFloorRef), ref, c);
  }

  // Cuts the lists to the CTA's K best windows, spread evenly over the warps.
  __device__ __forceinline__ void cut() {
    if (lane == 0) sh.count[warp] = listed;
    __syncthreads();
    uint64_t k[kListSlots];
    float ws[kListSlots];
    int have = 0;
#pragma unroll
    for (int j = 0; j < kListSlots; ++j) {
      const int f = j * kScanThreads + (int)threadIdx.x, w = f / kListWarp, i = f % kListWarp;
      const bool in = i < sh.count[w];
      k[j] = in ? sh.key[w][i] : 0;
      ws[j] = in ? sh.sum[w][i] : 0.0f;
      have += in;
    }
    int total;
    block_prefix(have, total, sh);
    const uint64_t t = total > K ? select_kth(k, K, sh) : 1;
    int keep = 0;
    uint32_t least = 0xFFFFFFFFu;
#pragma unroll
    for (int j = 0; j < kListSlots; ++j)
      if (k[j] >= t) {
        ++keep;
        least = min(least, (uint32_t)(k[j] >> 32));
      }
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    if (lane == 0) sh.redu[1][warp] = least;
    int at = block_prefix(keep, total, sh);
#pragma unroll
    for (int w = 0; w < kScanWarps; ++w) least = min(least, sh.redu[1][w]);
    if (total >= K) {
      // windows that are read from now on come after those of equal maximum
      if (unordered(least) > thr) raise(unordered(least));
      list_thr = unordered(ordered(thr) + 1);
      exact = true;
    }
#pragma unroll
    for (int j = 0; j < kListSlots; ++j) {
      if (k[j] >= t) {
        sh.key[at % kScanWarps][at / kScanWarps] = k[j];
        sh.sum[at % kScanWarps][at / kScanWarps] = ws[j];
        ++at;
      } else if (k[j]) {
        drop(k[j], ws[j]);
      }
    }
    listed = (total - warp + kScanWarps - 1) / kScanWarps;
    __syncthreads();
  }

  // Scans this CTA's part of row t for the k largest at 2^(z cc).
  __device__ __forceinline__ void scan(int t, int k, float cc) {
    const Row<T> row = row_of(t);
    slice(row, lo, hi);
    K = k;
    c = cc;
    thr = list_thr = top0 = top1 = -INFINITY;
    exact = false;
    ref = kFloorRef;
    s = lost = 0.0f;
    listed = 0;
    int refresh_at = 0;
    const int steps = max((hi - lo + kScanStep - 1) / kScanStep, 1);
    for (int step = 0; step < steps; ++step) {
      const int stage = wait();
      const int i0 = lo + step * kScanStep + warp * kWarpStep + lane;
      uint4 v[kScanUnroll];
      float wm[kScanUnroll];
#pragma unroll
      for (int u = 0; u < kScanUnroll; ++u) {
        const int i = i0 + 32 * u;
        const uint32_t none = neg_inf_bits(row.p);
        v[u] = make_uint4(none, none, none, none);
        if (i < hi) v[u] = row.whole(i) ? sh.ring[warp][stage][lane + 32 * u] : load_window(row, i);
        wm[u] = window_max<T>(v[u]);
      }
      top0 = fmaxf(top0, fmaxf(wm[0], wm[1]));
      top1 = fmaxf(top1, fmaxf(wm[2], wm[3]));
      issue();
      if (step == refresh_at || step + 1 == steps) {
        refresh();
        refresh_at = 2 * step + 1;
      }
      float sums = 0.0f;
#pragma unroll
      for (int u = 0; u < kScanUnroll; ++u) {
        const int i = i0 + 32 * u;
        const bool list = i < hi && wm[u] >= list_thr;
        const float r = list ? fmaxf(wm[u], kFloorRef) : ref;
        const float ws = window_sum<T>(v[u], c, r);
        const uint32_t mask = __ballot_sync(0xFFFFFFFFu, list);
        if (mask) {
          if (list) {
            const int at = listed + __popc(mask & ((1u << lane) - 1u));
            sh.key[warp][at] = make_key(wm[u], (uint32_t)i);
            sh.sum[warp][at] = ws;
          }
          listed += __popc(mask);
        }
        sums += list ? 0.0f : ws;
      }
      // s + sums with the rounding kept (a row's thread adds hundreds of these)
      const float y = sums - lost, z = s + y;
      lost = (z - s) - y;
      s = z;
      __syncwarp();
      if (step + 1 < steps && __syncthreads_or(listed > kListWarp - kWarpStep)) {
        refresh();
        if (__syncthreads_or(listed > kListWarp - kWarpStep)) cut();
      }
    }
    __syncthreads();
    if (lane == 0) sh.count[warp] = listed;
    __syncthreads();
    if (sh.late) s = NAN;
    int total = 0;
#pragma unroll
    for (int w = 0; w < kScanWarps; ++w) total += sh.count[w];
    if (total > kScanThreads) {
      __syncthreads();
      cut();
      if (lane == 0) sh.count[warp] = listed;
      __syncthreads();
    }
  }

  // The elements of the listed windows that reach the threshold, as keys (value,
  // id): written to dst in a fixed order, followed by zeros up to `fill`.
  // Returns their number, at most candidate_cap(K); if there were more, the K
  // largest alone.  All others go into s.
  __device__ __forceinline__ int candidates(int t, uint64_t *dst, int fill) {
    const Row<T> row = row_of(t);
    const int tid = threadIdx.x;
    uint64_t k[E] = {};
    int i = -1, left = tid, n = 0;
#pragma unroll
    for (int w = 0; w < kScanWarps; ++w) {
      if (left >= 0 && left < sh.count[w]) i = (int)key_index(sh.key[w][left]);
      left -= sh.count[w];
    }
    if (i >= 0) {
      float f[E];
      unpack<T>(load_window(row, i), f);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int id = i * E - row.mis + e;
        if (id >= 0 && id < vocab) {
          if (f[e] >= thr) {
            k[e] = make_key(f[e], (uint32_t)id);
            ++n;
          } else {
            s += exp_from(f[e], ref, c);
          }
        }
      }
    }
    return emit(k, n, exact ? K : candidate_cap(K), dst, fill);
  }
  template <int N>
  __device__ __forceinline__ int emit(uint64_t (&k)[N], int n, int most, uint64_t *dst, int fill) {
    int total;
    int at = block_prefix(n, total, sh);
    if (total > most) {
      exact = true;
      const uint64_t t = select_kth(k, K, sh);
      n = 0;
      uint32_t least = 0xFFFFFFFFu;
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (k[e] >= t) {
          ++n;
          least = min(least, (uint32_t)(k[e] >> 32));
        }
      least = __reduce_min_sync(0xFFFFFFFFu, least);
      if (lane == 0) sh.redu[1][warp] = least;
      at = block_prefix(n, total, sh);
#pragma unroll
      for (int w = 0; w < kScanWarps; ++w) least = min(least, sh.redu[1][w]);
      if (unordered(least) > thr) raise(unordered(least));
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (k[e] && k[e] < t) {
          s += exp_from(key_value(k[e]), ref, c);
          k[e] = 0;
        }
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (k[e]) dst[at++] = k[e];
    for (int i = total + (int)threadIdx.x; i < fill; i += kScanThreads) dst[i] = 0;
    return total;
  }

  // After scan(): gathers the cluster's candidates at the row's leader, which
  // changes from row to row (`turn`).  True there: then sh.cand holds n
  // candidates, the n largest elements of the row (n >= K unless the row has
  // fewer or NaN), and s (this thread's part), ref and thr are the row's.
  //
  // The barrier's phase of a row ends when all its parts are written.  A CTA
  // writes the next row's after that phase; a leader reads its row's before it
  // arrives at the next, and leads again a row later at the earliest, so that
  // one buffer is enough.
  __device__ __forceinline__ bool gather(int t, int turn, int &n) {
    if (C == 1) {
      n = candidates(t, sh.cand, 0);
      __syncthreads();
      return true;
    }
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, leader = turn % C, cap = candidate_cap(K);
    if (!waited) cluster_wait();
    candidates(t, cluster.map_shared_rank(recv, leader) + rank * recv_cap, cap);
    const float total = block_reduce<kScanThreads>(s, sh.redf, OpAdd());
    if (tid == 0) {
      *cluster.map_shared_rank(&sh.part_sum[rank], leader) = total;
      *cluster.map_shared_rank(&sh.part_thr[rank], leader) = thr;
      *cluster.map_shared_rank(&sh.part_exact[rank], leader) = exact;
    }
    cluster_arrive();
    waited = rank == leader;
    if (!waited) return false;
    cluster_wait();
    for (int i = 0; i < C; ++i) {
      thr = fmaxf(thr, sh.part_thr[i]);
      exact |= sh.part_exact[i] != 0;
    }
    ref = fmaxf(thr, kFloorRef);
    s = tid < C ? sh.part_sum[tid] * exp_from(fmaxf(sh.part_thr[tid], kFloorRef), ref, c) : 0.0f;
    uint64_t k[kTopMax * kClusterMax / kScanThreads];
    int mine = 0;
#pragma unroll
    for (int j = 0; j < kTopMax * kClusterMax / kScanThreads; ++j) {
      const int i = j * kScanThreads + tid, r = i / cap;
      k[j] = r < C ? recv[r * recv_cap + i % cap] : 0;
      if (k[j] && key_value(k[j]) < thr) {
        s += exp_from(key_value(k[j]), ref, c);
        k[j] = 0;
      }
      mine += k[j] != 0;
    }
    n = emit(k, mine, exact ? K : cap, sh.cand, 0);
    __syncthreads();
    return true;
  }
  // No CTA ends while another may write to its shared memory, or a copy to its own.
  __device__ __forceinline__ void finish() {
    if (!waited) cluster_wait();
    waited = true;
    if (dead)
      for (; used != issued; ++used)
        wait_copy(smem_u32(&sh.bar[warp][used % kScanStages]), (used / kScanStages) & 1);
  }
  bool waited;  // this thread has passed the last phase that it arrived at
  static __device__ __forceinline__ void cluster_arrive() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  }
  static __device__ __forceinline__ void cluster_wait() {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
};
#endif  // __CUDACC__

}  // namespace slimwise
