// norm.cu -- layer norm and RMS norm of rows, and their gradients.
//
//   mu = mean x (RMS: 0),  r = 1 / sqrt(mean (x - mu)^2 + eps),  n = (x - mu) r
//   y  = n g + b
//   g' = dy g,  dx = r (g' - mean g' - n mean(n g'))   (RMS: without mean g')
//   dg = sum over rows of dy n,  db = sum over rows of dy
//
// Both directions are bound by memory: the forward pass reads and writes a row
// once, the gradient reads two and writes one.  A row is dealt to a group of
// threads that holds it in registers from its load to its store; the group's
// sums go over shuffles and, above a warp, shared memory.  The variance is taken
// of differences from the mean, in registers, so that a mean far above the
// spread costs nothing of it.
//
// The gradient of the weight: a thread keeps the same columns for all rows of
// its CTA, so dg and db stay in its registers (32 columns of a thread: in shared
// memory) until the CTA's last row; a second kernel adds the CTAs' sums in order.
#include "train.cuh"

namespace slimwise {

namespace {

// Threads of a row and elements of a thread: rows up to 256, 1024, 2048, 4096,
// 8192 and 16384 long.  CTAs hold eight rows' groups of a warp, else one row's.
constexpr int kWarpRows = 8;
template <int TPR>
constexpr int kBlock = TPR == 32 ? 32 * kWarpRows : TPR;
// Rows loaded at once by a group: 16 (32: the longest rows) KB of a tensor in
// flight in 512 threads.
template <typename T, int N>
constexpr int kBatch = N >= 32 ? 1 : N == 16 ? (sizeof(T) == 2 ? 2 : 1) : (sizeof(T) == 2 ? 4 : 2);

// Sums of K values over the group's threads, known to all of them.  `buf` holds
// two sets of K values a warp, used in turn (`turn`), so that one barrier a
// reduction is enough.
template <int TPR, int K>
__device__ __forceinline__ void group_sum(float (&v)[K], float *buf, int &turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = warp_sum(v[k]);
  if constexpr (TPR > 32) {
    constexpr int W = TPR / 32;
    float *set = buf + turn * K * W;
    turn ^= 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) set[k * W + warp] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += set[k * W + w];
      v[k] = s;
    }
  }
}

struct NormArgs {
  int rows, hidden;
  int64_t stride, y_stride;
  const float *weight, *bias;
  float eps;
  float *mean, *rstd;
};

// R: rows that a group takes at once.
template <typename T, int V, int TPR, int N, int R, bool kLayer>
__global__ void __launch_bounds__(kBlock<TPR>)
    norm_kernel(const T *__restrict__ x, NormArgs a, T *__restrict__ y) {
  __shared__ float buf[2 * R * (TPR / 32)];
  int turn = 0;
  const int t = threadIdx.x % TPR;
  const int groups = gridDim.x * (kBlock<TPR> / TPR);
  const float inv = 1.0f / (float)a.hidden;
  for (int r0 = (blockIdx.x * (kBlock<TPR> / TPR) + threadIdx.x / TPR) * R; r0 < a.rows;
       r0 += groups * R) {
    RowPart<T, V, N> part[R];
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (r0 + i < a.rows) part[i].load(x + (int64_t)(r0 + i) * a.stride, t, TPR, a.hidden);
    float mu[R], q[R];
    if constexpr (kLayer) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        mu[i] = 0.0f;
        if (r0 + i < a.rows)
#pragma unroll
          for (int e = 0; e < N; ++e) mu[i] += part[i].get(e);
      }
      group_sum<TPR>(mu, buf, turn);
#pragma unroll
      for (int i = 0; i < R; ++i) mu[i] *= inv;
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      q[i] = 0.0f;
      if (r0 + i < a.rows)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          float d = part[i].get(e);
          if constexpr (kLayer)
            d = RowPart<T, V, N>::column(e, t, TPR) < a.hidden ? d - mu[i] : 0.0f;
          q[i] = fmaf(d, d, q[i]);
        }
    }
    group_sum<TPR>(q, buf, turn);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      q[i] = 1.0f / sqrtf(fmaf(q[i], inv, a.eps));
      if (t == 0 && r0 + i < a.rows) {
        a.rstd[r0 + i] = q[i];
        if (kLayer && a.mean) a.mean[r0 + i] = mu[i];
      }
    }
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      float g[2], b[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int c = RowPart<T, V, N>::column(e + j, t, TPR);
        g[j] = c < a.hidden ? __ldg(a.weight + c) : 0.0f;
        b[j] = a.bias && c < a.hidden ? __ldg(a.bias + c) : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (r0 + i >= a.rows) continue;
        float n[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          n[j] = part[i].get(e + j);
          if constexpr (kLayer) n[j] -= mu[i];
          n[j] = fmaf(n[j] * q[i], g[j], b[j]);
        }
        part[i].set2(e, n[0], n[1]);
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (r0 + i < a.rows) part[i].store(y + (int64_t)(r0 + i) * a.y_stride, t, TPR, a.hidden);
  }
}

struct GradArgs {
  int rows, hidden;
  int64_t dy_stride, stride, dx_stride;
  const float *weight, *mean, *rstd;
  float *partial;  // [CTAs][kLayer ? 2 : 1][hidden]
};

template <typename T, int V, int TPR, int N, bool kLayer>
__global__ void __launch_bounds__(kBlock<TPR>, 512 / kBlock<TPR>)
    norm_grad_kernel(const T *__restrict__ dy, const T *__restrict__ x, GradArgs a,
                     T *__restrict__ dx) {
  constexpr int R = kBatch<T, N>, K = kLayer ? 2 * R : R;
  constexpr int kGroups = kBlock<TPR> / TPR;
  constexpr bool kShared = N >= 32;
  using Part = RowPart<T, V, N>;
  __shared__ float buf[2 * K * (TPR / 32)];
  extern __shared__ float held[];  // kShared: dg [N][TPR], db [N][TPR]; groups of a warp: one group's sums
  int turn = 0;
  const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const float inv = 1.0f / (float)a.hidden;
  float g[N], dg[N], db[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int c = Part::column(e, t, TPR);
    g[e] = c < a.hidden ? __ldg(a.weight + c) : 0.0f;
    dg[e] = db[e] = 0.0f;
    if constexpr (kShared) {
      held[e * TPR + t] = 0.0f;
      if constexpr (kLayer) held[(N + e) * TPR + t] = 0.0f;
    }
  }
  for (int r0 = (blockIdx.x * kGroups + group) * R; r0 < a.rows; r0 += gridDim.x * kGroups * R) {
    Part d[R], p[R];
    float mu[R], rs[R], s[K];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const bool in = r0 + i < a.rows;
      if (in) {
        d[i].load(dy + (int64_t)(r0 + i) * a.dy_stride, t, TPR, a.hidden);
        p[i].load(x + (int64_t)(r0 + i) * a.stride, t, TPR, a.hidden);
      } else {
#pragma unroll
        for (int k = 0; k < Part::kWords; ++k) d[i].w[k] = p[i].w[k] = 0u;
      }
      rs[i] = in ? __ldg(a.rstd + r0 + i) : 0.0f;
      mu[i] = kLayer && in ? __ldg(a.mean + r0 + i) : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = 0.0f;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        // (columns past the row: dy = 0 and g = 0)
        const float de = d[i].get(e), n = (p[i].get(e) - mu[i]) * rs[i], ge = de * g[e];
        s[i] = fmaf(n, ge, s[i]);
        if constexpr (kLayer) s[R + i] += ge;
        if constexpr (kShared) {
          held[e * TPR + t] = fmaf(de, n, held[e * TPR + t]);
          if constexpr (kLayer) held[(N + e) * TPR + t] += de;
        } else {
          dg[e] = fmaf(de, n, dg[e]);
          if constexpr (kLayer) db[e] += de;
        }
      }
    group_sum<TPR>(s, buf, turn);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (r0 + i >= a.rows) continue;
      const float m = s[i] * inv, m0 = kLayer ? s[R + i] * inv : 0.0f;
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        float v[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float n = (p[i].get(e + j) - mu[i]) * rs[i];
          v[j] = rs[i] * (fmaf(d[i].get(e + j), g[e + j], -m0) - n * m);
        }
        p[i].set2(e, v[0], v[1]);
      }
      p[i].store(dx + (int64_t)(r0 + i) * a.dx_stride, t, TPR, a.hidden);
    }
  }
  // the CTA's sums: its groups' in turn
  float *out = a.partial + (int64_t)blockIdx.x * (kLayer ? 2 : 1) * a.hidden;
  if constexpr (kGroups > 1) {
    for (int k = 0; k < kGroups; ++k) {
      if (group == k) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          held[e * TPR + t] = (k ? held[e * TPR + t] : 0.0f) + dg[e];
          if constexpr (kLayer) held[(N + e) * TPR + t] = (k ? held[(N + e) * TPR + t] : 0.0f) + db[e];
        }
      }
      __syncthreads();
    }
    if (group != 0) return;
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int c = Part::column(e, t, TPR);
    if (c >= a.hidden) continue;
    out[c] = kShared || kGroups > 1 ? held[e * TPR + t] : dg[e];
    if constexpr (kLayer) out[a.hidden + c] = kShared || kGroups > 1 ? held[(N + e) * TPR + t] : db[e];
  }
}

// The CTAs' sums of each column, in the order of the CTAs: eight parts of them,
// each in order, then the parts.
// (`partial` is still written when this kernel starts: no __restrict__)
__global__ void __launch_bounds__(256)
    norm_grad_sum_kernel(const float *partial, int ctas, int columns, int hidden, float *dweight,
                         float *dbias) {
  __shared__ float part[8][32];
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  pdl_wait_primary();
  float s = 0.0f;
  if (c < columns) {
    const int per = (ctas + 7) / 8, end = min(ctas, (k + 1) * per);
#pragma unroll 8
    for (int i = k * per; i < end; ++i) s += partial[(int64_t)i * columns + c];
  }
  part[k][lane] = s;
  __syncthreads();
  if (k == 0 && c < columns) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += part[i][lane];
    if (c < hidden) dweight[c] = s;
    else if (dbias) dbias[c - hidden] = s;
  }
}

int grad_ctas(int rows, int hidden) {
  const int tpr = hidden <= 256 ? 32 : hidden <= 1024 ? 128 : hidden <= 2048 ? 256 : 512;
  const int groups = tpr == 32 ? kWarpRows : 1, most = kSms * (512 / (tpr * groups));
  // (at least a row for every group)
  const int ctas = (rows + groups - 1) / groups;
  return ctas < most ? ctas : most;
}

template <typename T, int V, int TPR, int N, bool kLayer>
cudaError_t norm_rows(const T *x, const NormArgs &a, T *y, cudaStream_t stream) {
  constexpr int R = kBatch<T, N>, kGroups = kBlock<TPR> / TPR;
  // few rows: one at a time, on as many SMs as there are
  const int64_t most = (int64_t)kSms * (2048 / kBlock<TPR>);
  if (R == 1 || a.rows < (int64_t)kSms * kGroups * R) {
    const int64_t ctas = ((int64_t)a.rows + kGroups - 1) / kGroups;
    norm_kernel<T, V, TPR, N, 1, kLayer>
        <<<(unsigned)(ctas < most ? ctas : most), kBlock<TPR>, 0, stream>>>(x, a, y);
  } else {
    const int64_t ctas = ((int64_t)a.rows + kGroups * R - 1) / (kGroups * R);
    norm_kernel<T, V, TPR, N, R, kLayer>
        <<<(unsigned)(ctas < most ? ctas : most), kBlock<TPR>, 0, stream>>>(x, a, y);
  }
  return cudaGetLastError();
}

template <typename T, int V, int TPR, int N, bool kLayer>
cudaError_t grad_rows(const T *dy, const T *x, const GradArgs &a, T *dx, float *dweight,
                      float *dbias, cudaStream_t stream) {
  constexpr bool kHeld = N >= 32 || kBlock<TPR> > TPR;
  constexpr size_t smem = kHeld ? (size_t)(kLayer ? 2 : 1) * N * TPR * 4 : 0;
  auto kernel = norm_grad_kernel<T, V, TPR, N, kLayer>;
  if (smem > 48 * 1024) {
    const cudaError_t err =
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (err != cudaSuccess) return err;
  }
  const int ctas = grad_ctas(a.rows, a.hidden);
  kernel<<<ctas, kBlock<TPR>, smem, stream>>>(dy, x, a, dx);
  const cudaError_t err = cudaGetLastError();
  if (err != cudaSuccess) return err;
  const int columns = (kLayer ? 2 : 1) * a.hidden;
  return launch_chained(norm_grad_sum_kernel, dim3((columns + 31) / 32), dim3(256), 0, stream, 1,
                        true, a.partial, ctas, columns, a.hidden, dweight, dbias);
}

// Calls f.template operator()<T, V, TPR, N>() for a row's type, access and length.
template <typename F>
cudaError_t dispatch(int dtype, int v, int hidden, F &&f) {
#define SLIMWISE_LENGTHS(T, V)                                        \
  return hidden <= 256    ? f.template operator()<T, V, 32, 8>()      \
         : hidden <= 1024 ? f.template operator()<T, V, 128, 8>()     \
         : hidden <= 2048 ? f.template operator()<T, V, 256, 8>()     \
         : hidden <= 4096 ? f.template operator()<T, V, 512, 8>()     \
         : hidden <= 8192 ? f.template operator()<T, V, 512, 16>()    \
                          : f.template operator()<T, V, 512, 32>()
  if (dtype == SLIMWISE_DTYPE_BF16) {
    if (v == 8) SLIMWISE_LENGTHS(__nv_bfloat16, 8);
    if (v == 2) SLIMWISE_LENGTHS(__nv_bfloat16, 2);
    SLIMWISE_LENGTHS(__nv_bfloat16, 1);
  }
  if (v == 4) SLIMWISE_LENGTHS(float, 4);
  SLIMWISE_LENGTHS(float, 1);
#undef SLIMWISE_LENGTHS
}

template <bool kLayer>
struct NormCall {
  const void *x;
  NormArgs a;
  void *y;
  cudaStream_t stream;
  template <typename T, int V, int TPR, int N>
  cudaError_t operator()() const {
    return norm_rows<T, V, TPR, N, kLayer>(static_cast<const T *>(x), a, static_cast<T *>(y), stream);
  }
};

template <bool kLayer>
struct GradCall {
  const void *dy, *x;
  GradArgs a;
  void *dx;
  float *dweight, *dbias;
  cudaStream_t stream;
  template <typename T, int V, int TPR, int N>
  cudaError_t operator()() const {
    return grad_rows<T, V, TPR, N, kLayer>(static_cast<const T *>(dy), static_cast<const T *>(x), a,
                                           static_cast<T *>(dx), dweight, dbias, stream);
  }
};

}  // namespace

cudaError_t launch_norm(const void *x, int dtype, int rows, int hidden, int64_t stride,
                        const float *weight, const float *bias, bool layer, float eps, void *y,
                        int64_t y_stride, float *mean, float *rstd, cudaStream_t stream) {
  const void *base[2] = {x, y};
  const int64_t strides[2] = {stride, y_stride};
  const int v = row_vector(dtype == SLIMWISE_DTYPE_BF16 ? 2 : 4, hidden, 2, base, strides);
  const NormArgs a = {rows, hidden, stride, y_stride, weight, bias, eps, mean, rstd};
  return layer ? dispatch(dtype, v, hidden, NormCall<true>{x, a, y, stream})
               : dispatch(dtype, v, hidden, NormCall<false>{x, a, y, stream});
}

size_t norm_grad_workspace(int rows, int hidden) {
  return (size_t)grad_ctas(rows, hidden) * 2 * hidden * sizeof(float);
}

cudaError_t launch_norm_grad(const void *dy, int64_t dy_stride, const void *x, int dtype, int rows,
                             int hidden, int64_t stride, const float *weight, const float *mean,
                             const float *rstd, void *dx, int64_t dx_stride, float *dweight,
                             float *dbias, void *workspace, cudaStream_t stream) {
  const void *base[3] = {dy, x, dx};
  const int64_t strides[3] = {dy_stride, stride, dx_stride};
  const int v = row_vector(dtype == SLIMWISE_DTYPE_BF16 ? 2 : 4, hidden, 3, base, strides);
  const GradArgs a = {rows, hidden, dy_stride, stride, dx_stride, weight, mean, rstd,
                      static_cast<float *>(workspace)};
  return mean ? dispatch(dtype, v, hidden, GradCall<true>{dy, x, a, dx, dweight, dbias, stream})
              : dispatch(dtype, v, hidden, GradCall<false>{dy, x, a, dx, dweight, dbias, stream});
}

}  // namespace slimwise
