// train.cuh -- what the operators around the layer share (embedding, norm and
// the head's cross entropy, each with its gradient): rows of bf16 or fp32 at any
// start and stride in registers, and the launch of a chain of kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "common.cuh"

namespace slimwise {

constexpr int kEmbedVocabMax = 1 << 20;  // rows of an embedding table
constexpr int kRowMax = 16384;           // longest row of the norm and the embedding
constexpr int kSms = 152;                // SMs that persistent grids are made for

// Launches a kernel as the one before it on the stream ends (programmatic
// dependent launch): it waits with pdl_wait_primary() before it touches memory.
// smem above 48 KB: allowed by the caller (cudaFuncSetAttribute).
template <typename... P, typename... A>
inline cudaError_t launch_chained(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem,
                                  cudaStream_t stream, int cluster, bool chained, A... args) {
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (chained) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)cluster;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = (unsigned)n;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

// Lets `kernel` have `bytes` of dynamic shared memory on the current device, once for each
// device that `devices` has no bit of yet.
inline cudaError_t allow_shared(std::atomic<uint64_t> &devices, const void *kernel, int bytes) {
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (devices.load(std::memory_order_acquire) & bit) return cudaSuccess;
  err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (err == cudaSuccess) devices.fetch_or(bit, std::memory_order_release);
  return err;
}

// Elements that one access of rows may take: 16 bytes of them where every row
// starts on a 16-byte boundary and is a multiple of them long, else (bf16) two,
// else one.
inline int row_vector(int element_bytes, int hidden, int n, const void *const *base,
                      const int64_t *stride) {
  int v = 16 / element_bytes;
  for (; v > 1; v = v > 2 ? 2 : 1) {
    if (element_bytes == 4 && v == 2) continue;
    const uintptr_t bytes = (uintptr_t)(v * element_bytes);
    bool ok = hidden % v == 0;
    for (int i = 0; i < n; ++i)
      ok = ok && reinterpret_cast<uintptr_t>(base[i]) % bytes == 0 && stride[i] % v == 0;
    if (ok) break;
  }
  return v;
}

// Whether rows may be read and written 16 bytes at a time as they lie: all start on
// 16-byte boundaries and are multiples of them long.
inline bool rows_aligned(int element_bytes, int hidden, int n, const void *const *base,
                         const int64_t *stride) {
  const int v = 16 / element_bytes;
  bool ok = hidden % v == 0;
  for (int i = 0; i < n; ++i)
    ok = ok && reinterpret_cast<uintptr_t>(base[i]) % 16 == 0 && stride[i] % v == 0;
  return ok;
}

cudaError_t launch_norm(const void *x, int dtype, int rows, int hidden, int64_t stride,
                        const float *weight, const float *bias, bool layer, float eps, void *y,
                        int64_t y_stride, float *mean, float *rstd, cudaStream_t stream);
size_t norm_grad_workspace(int rows, int hidden);
cudaError_t launch_norm_grad(const void *dy, int64_t dy_stride, const void *x, int dtype, int rows,
                             int hidden, int64_t stride, const float *weight, const float *mean,
                             const float *rstd, void *dx, int64_t dx_stride, float *dweight,
                             float *dbias, void *workspace, cudaStream_t stream);

cudaError_t launch_embed(const void *table, int dtype, int vocab, int hidden, int64_t stride,
                         const int32_t *ids, int rows, float scale, void *out, int64_t out_stride,
                         cudaStream_t stream);
size_t embed_grad_workspace(int rows, int hidden);
cudaError_t launch_embed_grad(const void *grad, int dtype, int rows, int hidden, int64_t stride,
                              const int32_t *ids, float scale, void *out, int out_dtype, int vocab,
                              int64_t out_stride, bool accumulate, void *workspace,
                              cudaStream_t stream);

size_t linear_loss_workspace(int rows, int hidden, int vocab, bool grad_hidden, bool grad_weight);
struct LinearLossArgs {
  const void *hidden;
  int64_t hidden_stride;
  const void *weight;
  int64_t weight_stride;
  int rows, width, vocab;
  const int32_t *labels;
  const float *row_weight;
  float *row_loss, *loss;
  void *grad_hidden;
  int64_t grad_hidden_stride;
  void *grad_weight;
  int grad_weight_dtype;
  int64_t grad_weight_stride;
};
cudaError_t launch_linear_loss(const LinearLossArgs &a, void *workspace, cudaStream_t stream);

#if defined(__CUDACC__)
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&b);
}

// Two fp32 numbers in a register pair, and arithmetic on both at once.
struct F2 {
  uint64_t v;
};
__device__ __forceinline__ F2 f2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ F2 f2(float a) { return f2(a, a); }
__device__ __forceinline__ float2 halves(F2 a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}

// Where a matrix's elements lie: reads of rows stay inside.
struct Extent {
  uintptr_t lo, hi;
};
template <typename T>
__host__ __device__ inline Extent extent_of(const T *base, int64_t rows, int64_t stride, int hidden) {
  const uintptr_t b = reinterpret_cast<uintptr_t>(base);
  return {b, b + (rows ? (uintptr_t)((rows - 1) * stride + hidden) * sizeof(T) : 0)};
}

// A 16-byte window, element by element: what lies outside [lo, hi) is neither read
// (but 0) nor written.
template <typename T>
__device__ __noinline__ uint4 read_edge(uintptr_t window, uintptr_t lo, uintptr_t hi) {
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uintptr_t a = window + 4 * i;
    if constexpr (sizeof(T) == 4) {
      if (a >= lo && a < hi) w[i] = __ldcg(reinterpret_cast<const uint32_t *>(a));
    } else {
      if (a >= lo && a < hi) w[i] = __ldcg(reinterpret_cast<const unsigned short *>(a));
      if (a + 2 >= lo && a + 2 < hi) w[i] |= (uint32_t)__ldcg(reinterpret_cast<const unsigned short *>(a + 2)) << 16;
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __noinline__ void write_edge(uint4 v, uintptr_t window, uintptr_t lo, uintptr_t hi) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uintptr_t a = window + 4 * i;
    if constexpr (sizeof(T) == 4) {
      if (a >= lo && a < hi) *reinterpret_cast<uint32_t *>(a) = w[i];
    } else {
      if (a >= lo && a < hi) *reinterpret_cast<unsigned short *>(a) = (unsigned short)w[i];
      if (a + 2 >= lo && a + 2 < hi) *reinterpret_cast<unsigned short *>(a + 2) = (unsigned short)(w[i] >> 16);
    }
  }
}
// 16 bytes from byte `by` (0..15, whole elements) of two windows.
__device__ __forceinline__ uint4 shift_windows(uint4 a, uint4 b, int by) {
  const uint32_t x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint32_t y[6], z[5];
#pragma unroll
  for (int k = 0; k < 6; ++k) y[k] = by & 8 ? x[k + 2] : x[k];
#pragma unroll
  for (int k = 0; k < 5; ++k) z[k] = by & 4 ? y[k + 1] : y[k];
  const uint32_t sel = by & 2 ? 0x5432u : 0x3210u;
  return make_uint4(__byte_perm(z[0], z[1], sel), __byte_perm(z[1], z[2], sel), __byte_perm(z[2], z[3], sel),
                    __byte_perm(z[3], z[4], sel));
}

// The two windows of each of a thread's accesses to a row, and where its elements
// begin in the first.
template <typename T, int N>
struct Windows {
  static constexpr int V = 16 / sizeof(T);
  uint4 a[N / V], b[N / V];
  int by;
  __device__ __forceinline__ void load(const T *row, int t, int threads, int width, Extent x) {
    // windows of a row reach up to 16 bytes beyond it: only the matrix's first and last
    // rows have to look at each
    const uintptr_t start = reinterpret_cast<uintptr_t>(row);
    const bool inside = start >= x.lo + 16 && start + (uintptr_t)max(width, 0) * sizeof(T) + 32 <= x.hi;
    by = (int)(start & 15);
#pragma unroll
    for (int p = 0; p < N / V; ++p) {
      const int c = (p * threads + t) * V;
      const uintptr_t at = start + (intptr_t)c * (int)sizeof(T) - by;
      a[p] = b[p] = make_uint4(0, 0, 0, 0);
      if (inside) {
        if (c < width) {
          a[p] = __ldg(reinterpret_cast<const uint4 *>(at));
          b[p] = __ldg(reinterpret_cast<const uint4 *>(at) + 1);
        }
      } else if (c < width) {
        a[p] = read_edge<T>(at, x.lo, x.hi);
        b[p] = read_edge<T>(at + 16, x.lo, x.hi);
      }
    }
  }
};

// A thread's part of a row: N elements of T in pieces of V, the row's pieces
// dealt to `threads` threads in turn, as they lie in memory (a bf16 in half a
// register).  Element e is column ((e / V) threads + t) V + e % V.
template <typename T, int V, int N>
struct RowPart {
  static constexpr int kWords = N * (int)sizeof(T) / 4;
  uint32_t w[kWords];

  template <bool kAfter, typename W>
  static __device__ __forceinline__ W read(const W *p) {
    if constexpr (kAfter) return __ldcg(p);
    else return __ldg(p);
  }
  static __device__ __forceinline__ int column(int e, int t, int threads) {
    return ((e / V) * threads + t) * V + e % V;
  }
  // Columns from `width` on read as 0.  kAfter: what the row holds is of a kernel
  // that this one may have been launched beside, or is written by this one too,
  // so it is not read as constant memory.
  template <bool kAfter = false>
  __device__ __forceinline__ void load(const T *row, int t, int threads, int width) {
#pragma unroll
    for (int p = 0; p < N / V; ++p) {
      const int c = (p * threads + t) * V;
      const bool in = c < width;
      constexpr int B = V * (int)sizeof(T);
      if constexpr (B >= 16) {
#pragma unroll
        for (int q = 0; q < B / 16; ++q) {
          const uint4 v = in ? read<kAfter>(reinterpret_cast<const uint4 *>(row + c) + q) : make_uint4(0, 0, 0, 0);
          uint32_t *o = w + (B / 4) * p + 4 * q;
          o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
        }
      } else if constexpr (B == 8) {
        const uint2 v = in ? read<kAfter>(reinterpret_cast<const uint2 *>(row + c)) : make_uint2(0, 0);
        w[2 * p] = v.x; w[2 * p + 1] = v.y;
      } else if constexpr (B == 4) {
        w[p] = in ? read<kAfter>(reinterpret_cast<const uint32_t *>(row + c)) : 0u;
      } else {
        const uint32_t v = in ? read<kAfter>(reinterpret_cast<const unsigned short *>(row + c)) : 0u;
        if (p & 1) w[p / 2] |= v << 16;
        else w[p / 2] = v;
      }
    }
  }
  // The same of a row that starts anywhere and of any width (V: 16 bytes): its windows
  // on their way (Windows), then shifted into place.
  __device__ __forceinline__ void take(const Windows<T, N> &x, int t, int threads, int width) {
    static_assert(V * sizeof(T) == 16, "windows");
#pragma unroll
    for (int p = 0; p < N / V; ++p) {
      const int left = width - (p * threads + t) * V;
      const uint4 v = shift_windows(x.a[p], x.b[p], x.by);
      uint32_t *o = w + 4 * p;
      o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
      if (left < V) {  // elements past the row: 0
        const int bytes = left * (int)sizeof(T);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (4 * k >= bytes) o[k] = 0u;
          else if (4 * k + 2 >= bytes) o[k] &= 0xFFFFu;
        }
      }
    }
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
  // Two neighbouring elements, e even.
  __device__ __forceinline__ F2 get2(int e) const { return f2(get(e), get(e + 1)); }
  __device__ __forceinline__ void set2(int e, F2 v) {
    const float2 h = halves(v);
    set2(e, h.x, h.y);
  }
  __device__ __forceinline__ void set2(int e, float a, float b) {
    if constexpr (sizeof(T) == 4) {
      w[e] = __float_as_uint(a);
      w[e + 1] = __float_as_uint(b);
    } else {
      w[e / 2] = pack_bf16(a, b);  // the one rounding to the output's type
    }
  }
  __device__ __forceinline__ void store(T *row, int t, int threads, int width) const {
#pragma unroll
    for (int p = 0; p < N / V; ++p) {
      const int c = (p * threads + t) * V;
      if (c >= width) continue;
      constexpr int B = V * (int)sizeof(T);
      if constexpr (B >= 16) {
#pragma unroll
        for (int q = 0; q < B / 16; ++q) {
          const uint32_t *o = w + (B / 4) * p + 4 * q;
          reinterpret_cast<uint4 *>(row + c)[q] = make_uint4(o[0], o[1], o[2], o[3]);
        }
      } else if constexpr (B == 8) {
        *reinterpret_cast<uint2 *>(row + c) = make_uint2(w[2 * p], w[2 * p + 1]);
      } else if constexpr (B == 4) {
        *reinterpret_cast<uint32_t *>(row + c) = w[p];
      } else {
        *reinterpret_cast<unsigned short *>(row + c) = (unsigned short)(w[p / 2] >> (p & 1 ? 16 : 0));
      }
    }
  }
};
#endif  // __CUDACC__

}  // namespace slimwise
