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

#include <atomic>

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
// attribute, one value per kernel, set on its first launch on a device and again
// after a launch that failed (a context that was reset has lost it); smem: this
// launch's.
// Clusters of more than 8 CTAs are asked for with kWideClusters.
template <auto kKernel, bool kWideClusters = false, typename... A>
inline cudaError_t launch_clusters(int clusters, int C, int threads, size_t smem, size_t smem_max,
                                   cudaStream_t stream, A... args) {
  static std::atomic<uint64_t> ready{0};  // a bit for each device
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    err = cudaFuncSetAttribute(reinterpret_cast<const void *>(kKernel),
                               cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_max);
    if (err == cudaSuccess && kWideClusters)
      err = cudaFuncSetAttribute(reinterpret_cast<const void *>(kKernel),
                                 cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (err != cudaSuccess) return err;
    ready.fetch_or(bit, std::memory_order_release);
  }
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
  err = cudaLaunchKernelEx(&cfg, kKernel, args...);
  if (err != cudaSuccess) ready.fetch_and(~bit, std::memory_order_release);
  return err;
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

// How a scan for the K largest is launched: CTAs of a cluster (a row is split
// over them), clusters, each of which takes every clusters-th row, and which
// kernel: for kFewCtas CTAs of an SM if those hold all rows, else for kManyCtas.
// few_stages: of the few's rings; more_smem: the kernel's shared memory besides
// the scan's.
constexpr int kManyCtas = 4, kFewCtas = 3, kManyStages = 2;
struct ScanGrid {
  int C, clusters;
  bool few;
  size_t smem;
};
ScanGrid scan_grid(int rows, int vocab, int element_bytes, int room, int K, bool long_lists, int few_stages,
                   size_t more_smem);

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
  int whole_lo, whole_n;  // the windows that lie in the row: from, number
  __device__ __forceinline__ Row(const T *row, int V) : p(row), vocab(V) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(row);
    mis = (int)((a & 15) / sizeof(T));
    w = reinterpret_cast<const uint4 *>(a & ~(uintptr_t)15);
    windows = (mis + V + E - 1) / E;
    whole_lo = mis > 0;
    whole_n = max((mis + V) / E - whole_lo, 0);
  }
  __device__ __forceinline__ bool whole(int i) const { return (unsigned)(i - whole_lo) < (unsigned)whole_n; }
};

__device__ __forceinline__ uint32_t neg_inf_bits(const __nv_bfloat16 *) { return 0xFF80FF80u; }
__device__ __forceinline__ uint32_t neg_inf_bits(const float *) { return 0xFF800000u; }

__device__ __forceinline__ uint4 ld_global_v4(const uint4 *p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// Window i of the row, -inf outside the row.
template <typename T>
__device__ __forceinline__ uint4 load_window(const Row<T> &r, int i) {
  if (r.whole(i)) return ld_global_v4(r.w + i);
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

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }

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

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Of two windows (kNan: NaN if any is).
template <typename T, bool kNan>
__device__ __forceinline__ float window_max(const uint4 &v, const uint4 &w) {
  if constexpr (kNan && sizeof(T) == 4) {
    const uint32_t a[8] = {v.x, v.y, v.z, v.w, w.x, w.y, w.z, w.w};
    float m = __uint_as_float(a[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = max_nan(m, __uint_as_float(a[i]));
    return m;
  } else if constexpr (kNan) {
    const uint32_t m = max2_nan(max2_nan(max2_nan(v.x, w.x), max2_nan(v.y, w.y)),
                                max2_nan(max2_nan(v.z, w.z), max2_nan(v.w, w.w)));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
  } else if constexpr (sizeof(T) == 4) {
    return fmaxf(window_max<T>(v), window_max<T>(w));
  } else {
    uint4 m;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(m.x) : "r"(v.x), "r"(w.x));
    asm("max.bf16x2 %0, %1, %2;" : "=r"(m.y) : "r"(v.y), "r"(w.y));
    asm("max.bf16x2 %0, %1, %2;" : "=r"(m.z) : "r"(v.z), "r"(w.z));
    asm("max.bf16x2 %0, %1, %2;" : "=r"(m.w) : "r"(v.w), "r"(w.w));
    return window_max<T>(m);
  }
}

// Bulk copy of whole windows into shared memory, counted on an mbarrier.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
      "l"(src), "r"(bytes), "r"(bar)
      : "memory");
}
// Bulk copy of whole windows into L2.
__device__ __forceinline__ void bulk_prefetch(const void *src, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
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

// Sum over N windows of 2^((z - ref) c).
template <typename T, int N>
__device__ __forceinline__ float windows_sum(const uint4 (&v)[N], float c, float ref) {
  constexpr int P = 8 / (int)sizeof(T);
  const uint64_t mr = pair(-ref, -ref), cc = pair(c, c);
  uint64_t sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint64_t p[P];
    unpack_pairs<T>(v[i], p);
#pragma unroll
    for (int q = 0; q < P; ++q) p[q] = exp2_pair(p[q], mr, cc);
#pragma unroll
    for (int d = 1; d < P; d *= 2)
#pragma unroll
      for (int q = 0; q < P; q += 2 * d) p[q] = add2(p[q], p[q + d]);
    sum[i] = p[0];
  }
#pragma unroll
  for (int d = 1; d < N; d *= 2)
#pragma unroll
    for (int i = 0; i + d < N; i += 2 * d) sum[i] = add2(sum[i], sum[i + d]);
  float a, b;
  split(sum[0], a, b);
  return a + b;
}
template <typename T>
__device__ __forceinline__ float window_sum(const uint4 &v, float c, float ref) {
  const uint4 one[1] = {v};
  return windows_sum<T, 1>(one, c, ref);
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
// The row is cut into one run for each warp of the cluster, and a run into units
// of four windows (64 bytes), one a lane in each step.  Each thread keeps the
// largest element of its windows (for K > 96, of two groups of them).  If m =
// K / 8 groups of each warp of a CTA reach a value, K elements do, so the least
// over the warps of each one's m-th largest group bounds the K-th largest
// element from below.  With many more groups than K it is near it, however long
// the row: about 100 elements lie above it for K = 64.  It costs a warp m
// reductions and the CTA one barrier, after the 2nd, 8th, 32nd, ... step and the last.  A
// unit whose maximum reaches the threshold is listed with its sum; any other
// only adds its sum to the thread's.
//
// The K largest elements of a run lie in its K units of largest maximum (ties:
// lower index), since each of those holds an element that goes before every
// element of the others.  So a warp whose list fills (many equal values, or rows
// in rising order) cuts it to its K best units, and nothing that matters is lost.
//
// Sums are relative to the threshold, not to the maximum: what lies below the
// list keeps its precision however far the list rises above it.  Which thread
// adds what never depends on timing, so that results are the same on every run.
//
// Each warp streams its run through a ring of its own with asynchronous copies; a
// stage is copied again as soon as its windows are in registers, and the copies
// of the next row are under way while a row is finished.  (Bulk copies counted on
// mbarriers cost about 80 instructions a step to issue and await, these 20, and
// the scan is bound by its instructions.)
constexpr int kScanThreads = 256;
constexpr int kScanWarps = kScanThreads / 32;
constexpr int kUnit = 4;                      // windows of a unit
constexpr int kWarpStep = 32 * kUnit;         // windows of a warp in a step
constexpr uint32_t kStageBytes = kWarpStep * 16;
constexpr int kClusterMax = 8;
constexpr int kStage = 32;
// Candidates that a CTA holds to pick from if they are more than it passes on (K
// above 64: the groups are then no more than twice the K wanted, and a threshold
// lets 1.5 to 2 K through on most rows).  1181 rows of 22705 bf16 at K = 256 took
// 151 us through most_of_many(), 120 held, and take 89 with a window a lane, the
// warps' candidates behind their lists, and three CTAs on an SM.
constexpr int kWide = 3 * kTopMax;
static_assert(kTopMax <= kScanThreads, "a thread for each candidate");

// Candidates that a CTA passes on: the K best and others, if there are no more
// than this (else the K best alone).  A power of two.
__host__ __device__ inline int candidate_cap(int K) { return K <= 8 ? 64 : K <= 32 ? 128 : kTopMax; }
// Units that a warp's list has room for: K (64 at least), and what a threshold
// of the 8th step lists until the 32nd.
constexpr int kListSpare = 80;
__host__ __device__ inline int list_room(int K) { return (K <= 64 ? 64 : (K + 31) / 32 * 32) + kListSpare; }
// A listed unit: its key (maximum, index of its first window), its sum of
// 2^((z - maximum) c), and, by the time its sum is not needed any more, a window
// that reaches the threshold (not necessarily its own).
struct alignas(16) Listed {
  uint64_t key;
  float sum;
  int window;
};
// A warp's list.  kLong: for long lists, without the window and in 12 bytes, keys
// and then sums (with K = 256 three CTAs fit an SM, not two).
template <bool kLong>
struct UnitList {
  static constexpr int kBytes = kLong ? 12 : sizeof(Listed);
  unsigned char *p;
  int room;
  __device__ __forceinline__ Listed *entry(int i) const { return reinterpret_cast<Listed *>(p) + i; }
  __device__ __forceinline__ uint64_t *keys() const { return reinterpret_cast<uint64_t *>(p); }
  __device__ __forceinline__ float *sums() const { return reinterpret_cast<float *>(p + room * 8); }
  __device__ __forceinline__ uint64_t key(int i) const { return kLong ? keys()[i] : entry(i)->key; }
  __device__ __forceinline__ Listed get(int i) const {
    if constexpr (kLong) return {keys()[i], sums()[i], 0};
    else return *entry(i);
  }
  __device__ __forceinline__ void put(int i, const Listed &e) const {
    if constexpr (kLong) {
      keys()[i] = e.key;
      sums()[i] = e.sum;
    } else {
      *entry(i) = e;
    }
  }
};

template <int kStages>
struct alignas(128) ScanShared {
  uint4 ring[kScanWarps][kStages][kWarpStep];
  uint64_t cand[kTopMax];
  uint64_t red64[kScanWarps];
  union {
    uint64_t stage[kScanWarps][kStage];  // a warp's candidates before their place is known
    struct {
      uint32_t hist[256];
      float by_rank[kTopMax];
    };
  };
  float redf[kScanWarps];
  uint32_t redu[2][kScanWarps];
  alignas(16) float reach[2][kScanWarps], known[2][kScanWarps];  // by refresh, in turn
  int part[2][kScanWarps];
  int count[kScanWarps];
  int sel_digit, sel_above, sel_bin;
  float part_sum[2][kClusterMax], part_thr[2][kClusterMax];  // at a row's leader: each CTA's
  int part_exact[2][kClusterMax];
  // then  UnitList [warps], of `room` units
  //       uint64_t [cluster][cap]  in clusters, at a row's leader: each CTA's
  //                                candidates (in clusters of two, two of these)
};
// room: of a warp's list; K: the largest number of candidates asked for.
// long_lists: those of a Scan with kLong, and after all that what it holds of
// candidates that are too many to pass on.
inline size_t scan_smem(int stages, int room, int K, int C, bool long_lists) {
  return sizeof(ScanShared<1>) + (size_t)(stages - 1) * kScanWarps * kStageBytes +
         (size_t)kScanWarps * room * (long_lists ? UnitList<true>::kBytes : UnitList<false>::kBytes) +
         (C > 1 ? (size_t)(C > 4 ? C : 4) * candidate_cap(K) * 8 : 0) + (long_lists ? kWide * 8 : 0);
}

// The bits of v from bit `from` (up to 64) up.
__device__ __forceinline__ uint64_t high_bits(uint64_t v, int from) {
  return from >= 64 ? 0 : v >> from << from;
}

// Threshold such that exactly K of the keys in the block's registers (0: none)
// are at least it; more than K are not 0.  A radix selection from the highest
// bit in which they differ, 8 bits a pass, that ends when a whole bin is taken.
template <int N, typename S>
__device__ __forceinline__ uint64_t select_kth(const uint64_t (&k)[N], int K, S &sh) {
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
template <typename S>
__device__ __forceinline__ int block_prefix(int v, int &total, S &sh) {
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

// The m-th largest of the warp's values, for small m: the largest taken away in
// turn.  At least `low` (a value known to be reached by as many, or -inf).
__device__ __forceinline__ float warp_mth(float a, int m, float low) {
  uint32_t o = ordered(a);
  while (true) {
    const uint32_t h = __reduce_max_sync(0xFFFFFFFFu, o);
    const bool top = o == h;
    m -= __popc(__ballot_sync(0xFFFFFFFFu, top));
    if (m <= 0) return fmaxf(low, unordered(h));
    if (h <= ordered(-INFINITY)) return low;
    if (top) o = 0;
  }
}

// A value that at least m of the warp's 2 x 32 values a, b reach, and few more;
// -inf if fewer than m are above -inf.  `low`: a value that is known to be
// reached by as many, or -inf.  Bisection over the order of the values' bits,
// which masked logits of the type's lowest value do not stretch as they would
// the range of the values, down to steps of `grain` bits.
__device__ __forceinline__ float warp_reach(float a, float b, int m, float low, uint32_t grain) {
  const uint32_t all = 0xFFFFFFFFu;
  const uint32_t oa = ordered(a), ob = ordered(b), none = ordered(-INFINITY);
  auto count = [&](uint32_t x) { return __popc(__ballot_sync(all, oa >= x)) + __popc(__ballot_sync(all, ob >= x)); };
  uint32_t lo, hi = __reduce_max_sync(all, max(oa, ob));
  if (low > -INFINITY) {
    lo = ordered(low);
  } else {
    lo = __reduce_min_sync(all, min(oa > none ? oa : all, ob > none ? ob : all));
    if (lo == all) return -INFINITY;
  }
  if (count(lo) < m) return low;
  while (hi > lo + grain) {
    const uint32_t mid = lo + (hi - lo) / 2;
    const int n = count(mid);
    if (n >= m) {
      lo = mid;
      if (n <= m + m / 4) break;
    } else {
      hi = mid;
    }
  }
  return unordered(lo);
}

// Lanes that share a candidate in a pass over all n of them (a power of two).
__device__ __forceinline__ int candidate_lanes(int n) {
  return n <= 32 ? 8 : n <= 64 ? 4 : n <= 128 ? 2 : 1;
}

// kCluster: rows are split over the CTAs of a cluster (else the cluster is one CTA).
// kSumless: scan() can leave out the sums (of the 400 instructions of a step,
// 120); s is then 0, or NaN where the row has NaN.
// kLong: for K above 64, whose lists and candidates are long.  kStages: of a ring.
template <typename T, bool kCluster, bool kSumless, bool kLong, int kStages>
struct Scan {
  static constexpr int E = Row<T>::E;
  static constexpr uint32_t kGrain = sizeof(T) == 2 ? 0xFFFFu : 0x1FFFu;  // a bf16's step; 2^-10 of an fp32
  using Shared = ScanShared<kStages>;
  Shared &sh;
  UnitList<kLong> list;  // this warp's
  uint64_t *recv;
  uint64_t *wide;
  int room, recv_cap;  // of a warp's list; of a CTA's part of recv
  const T *logits;
  int64_t stride;
  int vocab, rows;
  int log_parts;                // warps of a cluster
  int C, rank, clusters;        // CTAs of a cluster, this CTA's place, clusters of the grid
  int lane, warp;
  // the next copy: of row next_t, with next_left steps to go; this lane's first
  // window is the next_i-th of next_n to copy
  int next_t, next_left, next_i, next_n;
  const uint4 *next_src;
  uint32_t put_at, get_at;      // this lane's places in the ring's first stage
  uint32_t stage;               // offset of the stage that is read next, and then copied
  // the row at hand
  int K;
  float c, thr;                 // scale of the exponents (log2 e / temperature); threshold
  float list_thr;               // maximum at which a window is listed: thr, or more
  float ref, s, lost;           // s, with its low part: sum of 2^((z - ref) c) of what is not listed
  float top0, top1;             // maxima of this thread's groups
  int listed;                   // windows in this warp's list
  int turn;                     // of reach and known
  bool exact;                   // the K best alone are known to be complete

  // list_rooms: units that a warp's list has room for (at least K + 32), K_most: the
  // largest K of all rows
  __device__ __forceinline__ Scan(Shared &shared, int list_rooms, int K_most, const T *z, int64_t st,
                                  int V, int n)
      : sh(shared), logits(z), stride(st), vocab(V), rows(n) {
    if constexpr (kCluster) {
      cg::cluster_group cluster = cg::this_cluster();
      C = (int)cluster.num_blocks();
      rank = (int)cluster.block_rank();
    } else {
      C = 1;
      rank = 0;
    }
    clusters = (int)gridDim.x / C;
    log_parts = 31 - __clz(C * kScanWarps);
    lane = threadIdx.x & 31;
    warp = threadIdx.x >> 5;
    room = list_rooms;
    recv_cap = candidate_cap(K_most);
    list = list_of(warp);
    recv = reinterpret_cast<uint64_t *>(list_of(kScanWarps).p);
    wide = kLong ? recv + (kCluster ? max(C, 4) * recv_cap : 0) : nullptr;
    put_at = smem_u32(&sh.ring[warp][0][lane]);
    stage = 0;
    // a lane's windows are read in an order that keeps 8 lanes off each other's banks
    get_at = smem_u32(&sh.ring[warp][0][lane * kUnit]) + ((lane >> 1) & (kUnit - 1)) * 16;
    turn = 0;
    next_t = (int)(blockIdx.x / C);
    next_row();
    for (int i = 0; i < kStages; ++i) issue();
    if constexpr (kCluster) cluster_arrive();  // every CTA runs before another writes to its shared memory
  }
  __device__ __forceinline__ UnitList<kLong> list_of(int w) const {
    return {reinterpret_cast<unsigned char *>(&sh + 1) + w * room * UnitList<kLong>::kBytes, room};
  }
  __device__ __forceinline__ Row<T> row_of(int t) const {
    return Row<T>(logits + (int64_t)t * stride, vocab);
  }
  // Windows of a run: whole units.
  __device__ __forceinline__ int run_windows(const Row<T> &row) const {
    return (((row.windows + (1 << log_parts) - 1) >> log_parts) + kUnit - 1) & ~(kUnit - 1);
  }
  // Run of this warp: its first window, their number (returns), and the steps
  // that every warp of the cluster takes.
  __device__ __forceinline__ int run(const Row<T> &row, int &first, int &steps) const {
    const int per = run_windows(row);
    steps = (per + kWarpStep - 1) / kWarpStep;
    first = min((rank * kScanWarps + warp) * per, row.windows);
    return min(per, row.windows - first);
  }
  // [a, b): the windows of the run that lie whole in the row.
  __device__ __forceinline__ void whole_part(const Row<T> &row, int first, int n, int &a, int &b) const {
    a = max(row.whole_lo - first, 0);
    b = min(row.whole_lo + row.whole_n - first, n);
  }

  __device__ __forceinline__ void next_row() {
    if (next_t >= rows) {
      next_left = 1 << 30;
      next_n = 0;
      return;
    }
    const Row<T> row = row_of(next_t);
    int first, a, b;
    const int n = run(row, first, next_left);
    whole_part(row, first, n, a, b);
    next_src = row.w + first + lane;
    next_i = lane - a;
    next_n = max(b - a, 0);
  }
  // Starts the copy of this warp's windows of the next step, the row's partial
  // windows left out.  The stage's windows have been read by all lanes.
  __device__ __forceinline__ void issue() {
    if (next_i - lane >= 0 && next_i - lane + kWarpStep <= next_n) {
#pragma unroll
      for (int u = 0; u < kUnit; ++u) copy_window(u);
    } else {
#pragma unroll
      for (int u = 0; u < kUnit; ++u)
        if ((unsigned)(next_i + 32 * u) < (unsigned)next_n) copy_window(u);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    if constexpr (kStages == 2) stage ^= kStageBytes;
    else stage = stage == (kStages - 1) * kStageBytes ? 0 : stage + kStageBytes;
    next_i += kWarpStep;
    next_src += kWarpStep;
    if (--next_left == 0) {
      next_t += clusters;
      next_row();
    }
  }
  __device__ __forceinline__ void copy_window(int u) const {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(put_at + stage + u * 512), "l"(next_src + 32 * u)
                 : "memory");
  }
  // Waits for the oldest copy, of all lanes.
  __device__ __forceinline__ void wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    __syncwarp();
  }

  static __device__ __forceinline__ float least_of(const float (&x)[kScanWarps]) {
    const float4 a = *reinterpret_cast<const float4 *>(x), b = *reinterpret_cast<const float4 *>(x + 4);
    return fminf(fminf(fminf(a.x, a.y), fminf(a.z, a.w)), fminf(fminf(b.x, b.y), fminf(b.z, b.w)));
  }
  // Raises the threshold to what the groups of all warps show, and drops the
  // listed units below it (unless it is not the last time and they are few).
  __device__ __forceinline__ void refresh(bool last) {
    const int m = (K + kScanWarps - 1) / kScanWarps;
    const float reach = m <= 12 ? warp_mth(fmaxf(top0, top1), m, thr) : warp_reach(top0, top1, m, thr, kGrain);
    turn ^= 1;
    if (lane == 0) {
      sh.reach[turn][warp] = reach;
      sh.known[turn][warp] = thr;
    }
    // (a warp that cut its list knows more than the others)
    const bool cuts = __syncthreads_or(exact);
    float low = least_of(sh.reach[turn]), known = thr;
    if (cuts) {
      exact = true;
#pragma unroll
      for (int w = 0; w < kScanWarps; ++w) known = fmaxf(known, sh.known[turn][w]);
    }
    low = fmaxf(low, known);
    if (low > thr) {
      raise(low);
      list_thr = fmaxf(list_thr, thr);
    }
    if (last || listed > 24) keep_from(thr > -INFINITY ? (uint64_t)ordered(thr) << 32 : 1);
  }
  // Keeps the units of this warp's list whose keys are at least t, in order, and
  // drops the others.
  __device__ __forceinline__ void keep_from(uint64_t t) {
    int out = 0;
    for (int base = 0; base < listed; base += 32) {
      const int i = base + lane;
      Listed e = {0, 0.0f, 0};
      if (i < listed) e = list.get(i);
      const bool yes = e.key >= t;
      const uint32_t mask = __ballot_sync(0xFFFFFFFFu, yes);
      if (yes) list.put(out + __popc(mask & ((1u << lane) - 1u)), e);
      else if (e.key) s += e.sum * exp_from(fmaxf(key_value(e.key), kFloorRef), ref, c);
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

  // Cuts this warp's list to its K best windows: the windows that it reads from
  // now on come after those of equal maximum.
  __device__ __forceinline__ void cut() {
    uint64_t low = 0, high = ~0ull;  // at least K keys reach low, fewer reach high
    while (high - low > 1) {
      const uint64_t mid = low + (high - low) / 2;
      int n = 0;
      for (int i = lane; i < listed; i += 32) n += list.key(i) >= mid;
      n = __reduce_add_sync(0xFFFFFFFFu, n);
      if (n >= K) low = mid;
      else high = mid;
      if (n == K) break;
    }
    uint32_t least = 0xFFFFFFFFu;
    for (int i = lane; i < listed; i += 32)
      if (list.key(i) >= low) least = min(least, (uint32_t)(list.key(i) >> 32));
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    if (unordered(least) > thr) raise(unordered(least));
    list_thr = unordered(ordered(thr) + 1);
    exact = true;
    keep_from(low);
  }

  // Scans this CTA's part of row t for the k largest at 2^(z cc).
  __device__ __forceinline__ void scan(int t, int k, float cc, bool sums) {
    const Row<T> row = row_of(t);
    int first, steps, a, b;
    const int n = run(row, first, steps);
    whole_part(row, first, n, a, b);
    K = k;
    c = cc;
    thr = list_thr = top0 = top1 = -INFINITY;
    exact = false;
    ref = kFloorRef;
    s = lost = 0.0f;
    listed = 0;
    int refresh_at = 1;
    bool nan = false;
    const int full_from = (a + kWarpStep - 1) / kWarpStep, full_to = b / kWarpStep;
    for (int step = 0; step < steps; ++step) {
      wait();
      const int at = step * kWarpStep + lane * kUnit;
      uint4 v[kUnit];
      if (step >= full_from && step < full_to) {
#pragma unroll
        for (int u = 0; u < kUnit; ++u) v[u] = ld_shared_v4((get_at ^ (u * 16)) + stage);
      } else {
#pragma unroll
        for (int u = 0; u < kUnit; ++u) {
          const int i = at + (((get_at >> 4) ^ u) & (kUnit - 1));
          const uint32_t none = neg_inf_bits(row.p);
          v[u] = make_uint4(none, none, none, none);
          if (i < n) v[u] = i >= a && i < b ? ld_shared_v4((get_at ^ (u * 16)) + stage) : load_window(row, first + i);
        }
      }
      const float m0 = window_max<T, kSumless>(v[0], v[1]), m1 = window_max<T, kSumless>(v[2], v[3]);
      if constexpr (kSumless) nan |= m0 != m0 || m1 != m1;
      top0 = fmaxf(top0, m0);
      top1 = fmaxf(top1, m1);
      __syncwarp();
      issue();
      if (step == refresh_at || step + 1 == steps) {
        refresh(step + 1 == steps);
        refresh_at = 4 * step + 3;
      }
      const float m = fmaxf(m0, m1);
      const bool yes = m >= list_thr && at < n;
      float sum = 0.0f;
      if (!kSumless || sums) {
        const float from = yes ? fmaxf(m, kFloorRef) : ref;
        sum = windows_sum<T, kUnit>(v, c, from);
        // s + sum with the rounding kept (a row's thread adds hundreds of these)
        const float y = (yes ? 0.0f : sum) - lost, z = s + y;
        lost = (z - s) - y;
        s = z;
      }
      const uint32_t mask = __ballot_sync(0xFFFFFFFFu, yes);
      if (mask) {
        if (yes) {
          const int to = listed + __popc(mask & ((1u << lane) - 1u));
          list.put(to, {make_key(m, (uint32_t)(first + at)), sum, 0});
        }
        listed += __popc(mask);
        __syncwarp();
        if (listed > room - 32 && step + 1 < steps) cut();
      }
    }
    if (kSumless && nan) s = NAN;
  }

  // The elements of the listed units that reach the threshold, as keys (value,
  // id): written to dst in a fixed order, followed by zeros up to `fill`.
  // Returns their number, at most `cap`; if there were more, the K largest
  // alone.  All others go into s.
  __device__ __forceinline__ int candidates(int t, uint64_t *dst, int cap, int fill) {
    if constexpr (kLong) return long_candidates(t, dst, cap, fill);
    const Row<T> row = row_of(t);
    const int most = exact ? K : cap;
    // The windows of this warp's units that reach, a lane each, noted with
    // the listed units; then the elements of those
    // windows, a lane each.  A warp's candidates are held until it is known where
    // they go (if they are too many to hold, the elements are read again).
    const int windows = listed * kUnit;
    float add = 0.0f;
    int hits = 0, held = 0;
#pragma unroll 2
    for (int base = 0; base < windows; base += 32) {
      const int i = base + lane;
      const int at = i < windows ? (int)key_index(list.key(i / kUnit)) + i % kUnit : row.windows;
      const uint32_t none = neg_inf_bits(row.p);
      uint4 v = make_uint4(none, none, none, none);
      if (at < row.windows) v = load_window(row, at);
      const bool hit = at < row.windows && window_max<T>(v) >= thr;
      const uint32_t mask = __ballot_sync(0xFFFFFFFFu, hit);
      const int to = hits + __popc(mask & ((1u << lane) - 1u));
      if (hit && to < room) list.entry(to)->window = at;
      if (!hit) add += window_sum<T>(v, c, ref);
      hits += __popc(mask);
    }
    __syncwarp();
    auto pass = [&](auto put, float &sum) {
      const int elements = hits <= room ? hits * E : 0;
#pragma unroll 2
      for (int base = 0; base < elements; base += 32) {
        const int i = base + lane;
        const int id = i < elements ? list.entry(i / E)->window * E - row.mis + i % E : -1;
        const bool in = id >= 0 && id < vocab;
        const float z = in ? to_float(row.p[id]) : 0.0f;
        const bool yes = in && z >= thr;
        const uint32_t mask = __ballot_sync(0xFFFFFFFFu, yes);
        if (yes) put(__popc(mask & ((1u << lane) - 1u)), z, id);
        else if (in) sum += exp_from(z, ref, c);
        held += __popc(mask);
      }
    };
    pass([&](int at, float z, int id) {
      if (held + at < kStage) sh.stage[warp][held + at] = make_key(z, (uint32_t)id);
    }, add);
    if (hits > room) held = 1 << 20;  // too many to note: too many in all
    turn ^= 1;
    if (lane == 0) {
      sh.part[turn][warp] = held;
      sh.count[warp] = listed;
    }
    __syncthreads();
    int before = 0, total = 0, units = 0;
#pragma unroll
    for (int w = 0; w < kScanWarps; ++w) {
      if (w < warp) before += sh.part[turn][w];
      total += sh.part[turn][w];
      units += sh.count[w];
    }
    if (total > most) return most_of_many(row, dst, most, fill, units);
    s += add;
    if (held <= kStage) {
      if (lane < held) dst[before + lane] = sh.stage[warp][lane];
    } else {
      held = 0;
      float again = 0.0f;
      pass([&](int at, float z, int id) { dst[before + held + at] = make_key(z, (uint32_t)id); }, again);
    }
    for (int i = total + (int)threadIdx.x; i < fill; i += kScanThreads) dst[i] = 0;
    return total;
  }

  // candidates() for long lists, most of whose windows hold some: a window a lane,
  // and a warp's candidates held behind its list.
  __device__ __forceinline__ int long_candidates(int t, uint64_t *dst, int cap, int fill) {
    const Row<T> row = row_of(t);
    const int most = exact ? K : cap;
    const int windows = listed * kUnit, hold = room - listed;
    uint64_t *const keys = list.keys() + listed;
    float add = 0.0f;
    int held = 0;
    for (int base = 0; base < windows; base += 32) {
      const int i = base + lane;
      const int at = i < windows ? (int)key_index(list.key(i / kUnit)) + i % kUnit : row.windows;
      const uint32_t none = neg_inf_bits(row.p);
      uint4 v = make_uint4(none, none, none, none);
      if (at < row.windows) v = load_window(row, at);
      const bool hit = at < row.windows && window_max<T>(v) >= thr;
      if (!hit) add += window_sum<T>(v, c, ref);
      if (!__any_sync(0xFFFFFFFFu, hit)) continue;
      float z[E];
      unpack<T>(v, z);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int id = at * E - row.mis + e;
        const bool in = hit && (unsigned)id < (unsigned)vocab, yes = in && z[e] >= thr;
        const uint32_t mask = __ballot_sync(0xFFFFFFFFu, yes);
        const int to = held + __popc(mask & ((1u << lane) - 1u));
        if (yes && to < hold) keys[to] = make_key(z[e], (uint32_t)id);
        if (in && !yes) add += exp_from(z[e], ref, c);
        held += __popc(mask);
      }
    }
    if (held > hold) held = 1 << 20;  // too many to hold: too many in all
    turn ^= 1;
    if (lane == 0) {
      sh.part[turn][warp] = held;
      sh.count[warp] = listed;
    }
    __syncthreads();
    int before = 0, total = 0, units = 0;
#pragma unroll
    for (int w = 0; w < kScanWarps; ++w) {
      if (w < warp) before += sh.part[turn][w];
      total += sh.part[turn][w];
      units += sh.count[w];
    }
    const bool many = total > most;
    if (total > kWide) return most_of_many(row, dst, most, fill, units);
    s += add;
    uint64_t *const to = many ? wide : dst;
    for (int i = lane; i < held; i += 32) to[before + i] = keys[i];
    if (!many) {
      for (int i = total + (int)threadIdx.x; i < fill; i += kScanThreads) dst[i] = 0;
      return total;
    }
    __syncthreads();
    constexpr int kKeys = kWide / kScanThreads;
    uint64_t k[kKeys];
    int mine = 0;
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
      const int i = j * kScanThreads + (int)threadIdx.x;
      k[j] = i < total ? wide[i] : 0;
      mine += i < total;
    }
    return emit(k, mine, most, dst, fill);
  }

  // candidates() where there are more than may be passed on (many equal values,
  // or a short row): the units are cut to the K best of the CTA, their windows
  // to the K best, and the elements of those to the K largest.
  __device__ __forceinline__ int most_of_many(const Row<T> &row, uint64_t *dst, int most, int fill,
                                              int units) {
    const int tid = threadIdx.x;
    if (units > kScanThreads) {
      constexpr int kSlots = (kScanWarps * (kTopMax + kListSpare) + kScanThreads - 1) / kScanThreads;
      uint64_t k[kSlots];
#pragma unroll
      for (int j = 0; j < kSlots; ++j) {
        const int f = j * kScanThreads + tid, of = f / room, i = f - of * room;
        k[j] = of < kScanWarps && i < sh.count[of] ? list_of(of).key(i) : 0;
      }
      const uint64_t low = select_kth(k, K, sh);
      exact = true;
      raise_to_least(k, low);
      keep_from(low);
      if (lane == 0) sh.count[warp] = listed;
      __syncthreads();
    }
    // a unit each thread
    int unit = -1, left = tid;
#pragma unroll
    for (int w = 0; w < kScanWarps; ++w) {
      if (left >= 0 && left < sh.count[w]) unit = (int)key_index(list_of(w).key(left));
      left -= sh.count[w];
    }
    uint64_t k[kUnit];
    int n = 0;
#pragma unroll
    for (int u = 0; u < kUnit; ++u) {
      k[u] = 0;
      if (unit >= 0 && unit + u < row.windows) {
        const uint4 v = load_window(row, unit + u);
        const float m = window_max<T>(v);
        if (m >= thr) {
          k[u] = make_key(m, (uint32_t)(unit + u));
          ++n;
        } else {
          s += window_sum<T>(v, c, ref);
        }
      }
    }
    int total;
    int at = block_prefix(n, total, sh);
    if (total > kScanThreads) {
      const uint64_t low = select_kth(k, K, sh);
      exact = true;
      raise_to_least(k, low);
      n = 0;
#pragma unroll
      for (int u = 0; u < kUnit; ++u) {
        if (k[u] >= low) {
          ++n;
        } else if (k[u]) {
          s += window_sum<T>(load_window(row, unit + u), c, ref);
          k[u] = 0;
        }
      }
      at = block_prefix(n, total, sh);
    }
    // a window each thread
#pragma unroll
    for (int u = 0; u < kUnit; ++u)
      if (k[u]) sh.hist[at++] = key_index(k[u]);
    __syncthreads();
    const int window = tid < total ? (int)sh.hist[tid] : -1;
    __syncthreads();
    uint64_t key[E] = {};
    n = 0;
    if (window >= 0) {
      const uint4 v = load_window(row, window);
      float z[E];
      unpack<T>(v, z);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int id = window * E - row.mis + e;
        if (id >= 0 && id < vocab) {
          if (z[e] >= thr) {
            key[e] = make_key(z[e], (uint32_t)id);
            ++n;
          } else {
            s += exp_from(z[e], ref, c);
          }
        }
      }
    }
    return emit(key, n, exact ? K : most, dst, fill);
  }
  // Raises the threshold to the least value of the block's keys from `low` up.
  template <int N>
  __device__ __forceinline__ void raise_to_least(const uint64_t (&k)[N], uint64_t low) {
    uint32_t least = 0xFFFFFFFFu;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (k[j] >= low) least = min(least, (uint32_t)(k[j] >> 32));
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    if (lane == 0) sh.redu[1][warp] = least;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kScanWarps; ++w) least = min(least, sh.redu[1][w]);
    __syncthreads();
    if (unordered(least) > thr) raise(unordered(least));
  }
  // Leaves the keys from t up and adds the others to s; returns how many are left.
  template <int N>
  __device__ __forceinline__ int drop_below(uint64_t t, uint64_t (&k)[N]) {
    int n = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (k[e] >= t) {
        n += k[e] != 0;
      } else if (k[e]) {
        s += exp_from(key_value(k[e]), ref, c);
        k[e] = 0;
      }
    }
    return n;
  }
  // Writes the threads' keys (n of this thread are not 0) to dst, in the
  // threads' order; if they are more than `most`, the K largest alone.
  template <int N>
  __device__ __forceinline__ int emit(uint64_t (&k)[N], int n, int most, uint64_t *dst, int fill) {
    int total;
    int at = block_prefix(n, total, sh);
    if (total > most) {
      exact = true;
      const uint64_t t = select_kth(k, K, sh);
      raise_to_least(k, t);
      n = drop_below(t, k);
      at = block_prefix(n, total, sh);
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (k[e]) dst[at++] = k[e];
    for (int i = total + (int)threadIdx.x; i < fill; i += kScanThreads) dst[i] = 0;
    return total;
  }

  // In a cluster, a row's parts are gathered at its leader, which changes from
  // row to row, and the leader joins them once it has scanned and passed on its
  // part of the next row, so that it waits for no one.  A phase of the cluster's
  // barrier ends when all parts of a row are written; a CTA writes the next
  // row's after that.  A leader reads its row's parts before it arrives at the
  // second next phase, and leads again after C rows: in clusters of two, whose
  // CTAs may then write a second row's parts too early, they go to a second
  // buffer.
  __device__ __forceinline__ int leader_of(int row_turn) const { return row_turn & (C - 1); }
  __device__ __forceinline__ int half_of(int row_turn) const { return C == 2 ? row_turn >> 1 & 1 : 0; }
  // After scan(): passes on this CTA's part of row t.
  __device__ __forceinline__ void push(int t, int row_turn) {
    cg::cluster_group cluster = cg::this_cluster();
    const int leader = leader_of(row_turn), half = half_of(row_turn), cap = candidate_cap(K);
    cluster_wait();
    candidates(t, cluster.map_shared_rank(recv, leader) + (half * C + rank) * recv_cap, cap, cap);
    const float total = block_reduce<kScanThreads>(s, sh.redf, OpAdd());
    if (threadIdx.x == 0) {
      *cluster.map_shared_rank(&sh.part_sum[half][rank], leader) = total;
      *cluster.map_shared_rank(&sh.part_thr[half][rank], leader) = thr;
      *cluster.map_shared_rank(&sh.part_exact[half][rank], leader) = exact;
    }
    cluster_arrive();
  }
  // At the leader, after the phase of its row: as candidates() in a cluster of
  // one, sh.cand then holds the n largest elements of the row (n >= K unless the
  // row has fewer or NaN), and s (this thread's part), ref and thr are the row's.
  __device__ __forceinline__ int merge(int row_turn, int k_, float cc) {
    const int tid = threadIdx.x, half = half_of(row_turn);
    K = k_;
    c = cc;
    const int cap = candidate_cap(K);
    thr = -INFINITY;
    exact = false;
    for (int i = 0; i < C; ++i) {
      thr = fmaxf(thr, sh.part_thr[half][i]);
      exact |= sh.part_exact[half][i] != 0;
    }
    ref = fmaxf(thr, kFloorRef);
    s = tid < C ? sh.part_sum[half][tid] * exp_from(fmaxf(sh.part_thr[half][tid], kFloorRef), ref, c) : 0.0f;
    constexpr int kKeys = kTopMax * kClusterMax / kScanThreads;
    uint64_t k[kKeys];
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
      const int i = j * kScanThreads + tid, r = i >> (31 - __clz(cap));
      k[j] = r < C ? recv[(half * C + r) * recv_cap + (i & (cap - 1))] : 0;
      if (k[j]) most = fmaxf(most, key_value(k[j]));
    }
    // the threads' largest show a threshold too
    const float reach = (K + kScanWarps - 1) / kScanWarps <= 12
                            ? warp_mth(most, (K + kScanWarps - 1) / kScanWarps, -INFINITY)
                            : warp_reach(most, -INFINITY, (K + kScanWarps - 1) / kScanWarps, -INFINITY, kGrain);
    turn ^= 1;
    if (lane == 0) sh.reach[turn][warp] = reach;
    __syncthreads();
    const float low = least_of(sh.reach[turn]);
    if (low > thr) raise(low);
    const int mine = drop_below(thr > -INFINITY ? (uint64_t)ordered(thr) << 32 : 1, k);
    const int n = emit(k, mine, exact ? K : cap, sh.cand, 0);
    __syncthreads();
    return n;
  }
  // The loop over this cluster's rows.  request(t, K, c, sums) says what row t is
  // scanned for; done(t, n) is called by all threads of a row's leader.
  template <typename R, typename D>
  __device__ __forceinline__ void rows_of_cluster(R request, D done) {
    int t = (int)(blockIdx.x / C);
    for (int row_turn = 0;; ++row_turn, t += clusters) {
      const bool more = t < rows;
      int at = -1, n = 0, k;
      float cc;
      if (more) {
        bool sums;
        request(t, k, cc, sums);
        scan(t, k, cc, sums);
      }
      if constexpr (!kCluster) {
        if (more) {
          n = candidates(t, sh.cand, candidate_cap(K), 0);
          __syncthreads();
          at = t;
        }
      } else {
        if (more) push(t, row_turn);
        else cluster_wait();
        if (row_turn > 0 && leader_of(row_turn - 1) == rank) {
          at = t - clusters;
          bool sums;
          request(at, k, cc, sums);
          n = merge(row_turn - 1, k, cc);
        }
      }
      if (at >= 0) done(at, n);
      if (!more) break;
    }
  }
  static __device__ __forceinline__ void cluster_arrive() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  }
  static __device__ __forceinline__ void cluster_wait() {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
};
#endif  // __CUDACC__

}  // namespace slimwise
