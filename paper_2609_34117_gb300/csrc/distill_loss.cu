// distill_loss.cu -- the distillation loss of SlimWise Sec. 3.3, Eq. 3, and its
// gradient: cross entropy on the label plus KL against the teacher's top-K
// log-probabilities with one bucket for the residual mass.
//
//   p = softmax(z), q = softmax(z / tau), S the teacher's ids, P_j = exp l_j,
//   r = exp log_rest, M = sum P_j + r, Q = sum_{i not in S} q_i
//   CE = -log p_y,  KL = sum_j P_j (l_j - log q_j) + r (log r - log Q)
//   L  = a CE + (1 - a) tau^2 KL
//   dL/dz_i = a (p_i - [i = y]) + (1 - a) tau (M q_i - (i in S ? P_i : r q_i / Q))
//
// Q is summed over the elements outside S, not taken as 1 - the list's mass,
// which a student that is nearly sure would cancel to nothing: a bit per
// element, set in shared memory before the row is read, takes the list's
// elements out of the sums.
//
// A cluster handles a row.  Each CTA has its part copied into shared memory, in
// chunks that are all asked for at once, and sums exponentials against a
// running maximum as they come; one exchange over the cluster gives every CTA
// the row's sums, and the gradient is computed from shared memory: one read and
// one write of the row, which bound the kernel.
#include "vocab.cuh"

namespace slimwise {

constexpr int kLossThreads = 256;
constexpr int kLossUnroll = 2;
constexpr int kChunk = kLossThreads * kLossUnroll;  // windows of a copy (8 KB)
constexpr int kSliceMax = 200 * 1024;               // bytes of a row that one CTA may hold
constexpr int kChunksMax = kSliceMax / (kChunk * 16);
static_assert(kTopMax <= kLossThreads, "one thread per list entry");

struct LossArgs {
  const int32_t *labels, *top_ids;
  const float *top_logp, *log_rest, *row_weight;
  float *row_loss;
  int vocab, K;
  float alpha, tau;
};

struct LossShared {
  uint64_t bar[kChunksMax];
  float part[kClusterMax][3];  // each CTA's: reference, sum for p, sum for q
  float red[kLossThreads / 32][5];
};

template <int N>
__device__ __forceinline__ void block_sums(float (&v)[N], LossShared &sh) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
    if ((threadIdx.x & 31) == 0) sh.red[threadIdx.x >> 5][i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0.0f;
    for (int w = 0; w < kLossThreads / 32; ++w) v[i] += sh.red[w][i];
  }
  __syncthreads();
}

__device__ __forceinline__ void store(float *p, float v) { *p = v; }
__device__ __forceinline__ void store(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// The window without the elements whose bits are set (-inf in their place).
template <typename T>
__device__ __forceinline__ uint4 without(uint4 v, uint32_t bits) {
  uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (sizeof(T) == 4) {
      if (bits >> q & 1) u[q] = 0xFF800000u;
    } else {
      if (bits >> (2 * q) & 1) u[q] = (u[q] & 0xFFFF0000u) | 0xFF80u;
      if (bits >> (2 * q + 1) & 1) u[q] = (u[q] & 0xFFFFu) | 0xFF800000u;
    }
  }
  return make_uint4(u[0], u[1], u[2], u[3]);
}

template <typename T>
__device__ __forceinline__ void store_window(T *g, const Row<T> &row, int i,
                                             const float (&f)[Row<T>::E]) {
  constexpr int E = Row<T>::E;
  const int id0 = i * E - row.mis;
  if (row.whole(i)) {
    uint4 v;
    if constexpr (sizeof(T) == 4) {
      v = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                     __float_as_uint(f[3]));
    } else {
      uint32_t u[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[q]) : "f"(f[2 * q + 1]), "f"(f[2 * q]));
      v = make_uint4(u[0], u[1], u[2], u[3]);
    }
    *reinterpret_cast<uint4 *>(g + id0) = v;
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (id0 + e >= 0 && id0 + e < row.vocab) store(g + id0 + e, f[e]);
  }
}

// kTemp: tau is not 1, so that p and q are two softmaxes.
template <typename T, bool kGrad, bool kTemp>
__global__ void __launch_bounds__(kLossThreads, 4)
    distill_loss_kernel(const T *logits, int64_t stride, LossArgs a, T *grad, int64_t grad_stride) {
  constexpr int E = Row<T>::E;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ LossShared sh;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, V = a.vocab;
  const int64_t t = blockIdx.x / C;
  const Row<T> row(logits + t * stride, V);
  const int per = (row.windows + C - 1) / C;
  const int lo = min(rank * per, row.windows), hi = min(lo + per, row.windows);
  const int id_lo = max(lo * E - row.mis, 0), id_hi = min(hi * E - row.mis, V);
  T *const g = kGrad ? grad + t * grad_stride : nullptr;
  // gradient rows that start like the logits' are written in whole windows
  const bool alike = kGrad && ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(row.p)) & 15) == 0;
  const int label = a.labels[t];
  if (label < 0) {  // not trained on
    if (rank == 0 && tid == 0) a.row_loss[t] = 0.0f;
    if constexpr (kGrad) {
      const float zero[E] = {};
      if (alike)
        for (int i = lo + tid; i < hi; i += kLossThreads) store_window(g, row, i, zero);
      else
        for (int id = id_lo + tid; id < id_hi; id += kLossThreads) store(g + id, 0.0f);
    }
    return;
  }

  uint4 *const slice = reinterpret_cast<uint4 *>(smem);
  uint32_t *const bits = reinterpret_cast<uint32_t *>(smem + (size_t)per * 16);
  const int chunks = (hi - lo + kChunk - 1) / kChunk;
  if (tid == 0) {
    for (int i = 0; i < chunks; ++i) mbar_init(smem_u32(&sh.bar[i]), 1);
    mbar_fence_init();
    for (int i = 0; i < chunks; ++i) {
      // the row's partial windows at its ends are left out
      int first = lo + i * kChunk, end = min(first + kChunk, hi);
      uint4 *dst = slice + i * kChunk;
      if (first == 0 && !row.whole(0)) {
        ++first;
        ++dst;
      }
      if (end == row.windows && end > first && !row.whole(end - 1)) --end;
      const uint32_t bytes = end > first ? (uint32_t)(end - first) * 16 : 0;
      mbar_arrive_expect_tx(smem_u32(&sh.bar[i]), bytes);
      if (bytes) bulk_load(smem_u32(dst), row.w + first, bytes, smem_u32(&sh.bar[i]));
    }
  }
  for (int i = tid; i < (hi - lo + 3) / 4; i += kLossThreads) bits[i] = 0;
  const int id = tid < a.K ? a.top_ids[t * a.K + tid] : -1;
  const float lp = tid < a.K ? a.top_logp[t * a.K + tid] : 0.0f;
  const bool bad = __syncthreads_or(id >= V) || label >= V;
  const bool listed = id >= 0 && !bad;
  const float z = listed ? to_float(row.p[id]) : -INFINITY;
  const float zy = to_float(row.p[bad ? 0 : label]);
  if (listed && id >= id_lo && id < id_hi) {
    const int i = (id + row.mis) / E - lo;
    atomicOr(&bits[i >> 2], 1u << ((i & 3) * 8 + (id + row.mis) % E));
  }
  __syncthreads();

  // sums of the exponentials outside the list, against the largest so far: s1
  // of 2^((z - ref) c1), and with a temperature s2 of 2^((z - ref) c2)
  const float c1 = kLog2e, c2 = kTemp ? kLog2e / a.tau : kLog2e;
  const unsigned char *const byte = reinterpret_cast<const unsigned char *>(bits);
  float s1 = 0.0f, s2 = 0.0f, ref = kFloorRef;
  bool came = true;
  for (int b = 0; b < chunks; ++b) {
    came = came && wait_copy(smem_u32(&sh.bar[b]), 0);
    uint4 v[kLossUnroll];
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < kLossUnroll; ++u) {
      const int i = b * kChunk + u * kLossThreads + tid;
      const uint32_t none = neg_inf_bits(row.p);
      v[u] = make_uint4(none, none, none, none);
      if (lo + i < hi) {
        if (row.whole(lo + i)) {
          v[u] = slice[i];
        } else {
          v[u] = load_window(row, lo + i);
          slice[i] = v[u];
        }
        const uint32_t mk = byte[i];
        if (mk) v[u] = without<T>(v[u], mk);
      }
      m = fmaxf(m, window_max<T>(v[u]));
    }
    const float n = fmaxf(ref, m);
    s1 *= exp_from(ref, n, c1);
    if constexpr (kTemp) s2 *= exp_from(ref, n, c2);
    ref = n;
#pragma unroll
    for (int u = 0; u < kLossUnroll; ++u) {
      s1 += window_sum<T>(v[u], c1, ref);
      if constexpr (kTemp) s2 += window_sum<T>(v[u], c2, ref);
    }
  }
  if (!came) s1 = s2 = NAN;
  // over the block, then over the cluster
  {
    const float top = block_reduce<kLossThreads>(ref, &sh.red[0][0], OpMax());
    s1 = block_reduce<kLossThreads>(s1 * exp_from(ref, top, c1), &sh.red[0][0], OpAdd());
    if constexpr (kTemp)
      s2 = block_reduce<kLossThreads>(s2 * exp_from(ref, top, c2), &sh.red[0][0], OpAdd());
    ref = top;
  }
  cluster.sync();  // every CTA of the cluster runs
  if (tid < C) {
    float *const p = cluster.map_shared_rank(&sh.part[rank][0], tid);
    p[0] = ref;
    p[1] = s1;
    p[2] = s2;
  }
  const float z_top = block_reduce<kLossThreads>(z, &sh.red[0][0], OpMax());
  cluster.sync();
  ref = fmaxf(z_top, kFloorRef);
  for (int r = 0; r < C; ++r) ref = fmaxf(ref, sh.part[r][0]);
  float rest1 = 0.0f, rest2 = 0.0f;
  for (int r = 0; r < C; ++r) {
    rest1 += sh.part[r][1] * exp_from(sh.part[r][0], ref, c1);
    if constexpr (kTemp) rest2 += sh.part[r][2] * exp_from(sh.part[r][0], ref, c2);
  }
  if constexpr (!kTemp) rest2 = rest1;
  const float e1 = exp_from(z, ref, c1), e2 = kTemp ? exp_from(z, ref, c2) : e1;
  const float P = listed ? expf(lp) : 0.0f;
  float sums[3] = {listed ? e1 : 0.0f, listed ? e2 : 0.0f, P};
  block_sums(sums, sh);
  const float lr = a.log_rest[t], r = expf(lr);
  const float total1 = bad ? NAN : rest1 + sums[0], total2 = bad ? NAN : kTemp ? rest2 + sums[1] : total1;
  const float M = sums[2] + r;
  const float w = a.row_weight ? a.row_weight[t] : 1.0f;
  const float beta = (1.0f - a.alpha) * a.tau;
  if (rank == 0) {
    const float l2 = log2f(total2);
    float kl[1] = {P > 0.0f ? P * (lp - ((z - ref) * c2 - l2) * kLn2) : 0.0f};
    block_sums(kl, sh);
    if (tid == 0) {
      const float ce = (log2f(total1) - (zy - ref) * c1) * kLn2;
      const float kr = r > 0.0f ? r * (lr - (log2f(rest2) - l2) * kLn2) : 0.0f;
      a.row_loss[t] = a.alpha * ce + beta * a.tau * (kl[0] + kr);
    }
  }
  if constexpr (kGrad) {
    // outside the list: A e1 + B e2 (B into A when there is one softmax)
    const float share = rest2 > 0.0f ? r / rest2 : 0.0f;
    float A = w * a.alpha / total1;
    float B = w * beta * (M / total2 - share);
    if constexpr (!kTemp) A += B;
    auto outside = [&](float x) {
      float v = A * exp_from(x, ref, c1);
      if constexpr (kTemp) v = fmaf(B, exp_from(x, ref, c2), v);
      return v;
    };
    if (alike) {
      for (int i = lo + tid; i < hi; i += kLossThreads) {
        constexpr int P = E / 2;
        uint64_t p[P];
        unpack_pairs<T>(slice[i - lo], p);
        float f[E];
#pragma unroll
        for (int q = 0; q < P; ++q) {
          const uint64_t mr = pair(-ref, -ref);
          uint64_t v = mul2(pair(A, A), exp2_pair(p[q], mr, pair(c1, c1)));
          if constexpr (kTemp) v = add2(v, mul2(pair(B, B), exp2_pair(p[q], mr, pair(c2, c2))));
          split(v, f[2 * q], f[2 * q + 1]);
        }
        store_window(g, row, i, f);
      }
    } else {
      __syncthreads();
      const T *const part = reinterpret_cast<const T *>(slice) + row.mis - lo * E;
      for (int i = id_lo + tid; i < id_hi; i += kLossThreads) store(g + i, outside(to_float(part[i])));
    }
    // then the list's elements and the label
    const bool y_listed = __syncthreads_or(listed && id == label);
    if (!bad && listed && id >= id_lo && id < id_hi) {
      const float on = id == label ? a.alpha : 0.0f;
      store(g + id, w * (a.alpha * (e1 / total1) - on + beta * (M * (e2 / total2) - P)));
    }
    if (!bad && tid == 0 && !y_listed && label >= id_lo && label < id_hi)
      store(g + label, outside(zy) - w * a.alpha);
  }
  // a copy that did not come in time may still come: not after this CTA's end
  if (!came)
    for (int b = 0; b < chunks; ++b) wait_copy(smem_u32(&sh.bar[b]), 0);
}

// loss = sum of weight x row loss: thread i adds its rows i, i + 1024, ... in
// order, in fp64, then a butterfly and the warps in turn: the same every time.
__global__ void __launch_bounds__(1024)
    loss_sum_kernel(const float *__restrict__ row_loss, const float *__restrict__ row_weight,
                    int rows, float *__restrict__ loss) {
  __shared__ double part[32];
  double s = 0.0;
  for (int t = threadIdx.x; t < rows; t += 1024)
    s += (double)row_loss[t] * (row_weight ? (double)row_weight[t] : 1.0);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 32; ++w) s += part[w];
    *loss = (float)s;
  }
}

template <typename T, bool kGrad, bool kTemp>
static cudaError_t launch(const void *logits, int rows, int64_t stride, const LossArgs &a,
                          void *grad, int64_t grad_stride, cudaStream_t stream) {
  constexpr int E = Row<T>::E;
  const int windows = (a.vocab + 2 * E - 2) / E;  // the most that a row can cover
  int C = 1;
  while (C < kClusterMax && (windows > C * 40 * 64 || (rows * C < 608 && windows >= 2 * C * kChunk))) C *= 2;
  const size_t per = (size_t)(windows + C - 1) / C;
  const size_t smem = per * 16 + (per + 3) / 4 * 4;
  return launch_clusters(distill_loss_kernel<T, kGrad, kTemp>, rows, C, kLossThreads, smem,
                         kSliceMax + kSliceMax / 16, stream, static_cast<const T *>(logits),
                         stride, a, static_cast<T *>(grad), grad_stride);
}

template <typename T>
static cudaError_t launch(const void *logits, int rows, int64_t stride, const LossArgs &a,
                          void *grad, int64_t grad_stride, cudaStream_t stream) {
  const bool temp = a.tau != 1.0f;
  return grad ? temp ? launch<T, true, true>(logits, rows, stride, a, grad, grad_stride, stream)
                     : launch<T, true, false>(logits, rows, stride, a, grad, grad_stride, stream)
         : temp ? launch<T, false, true>(logits, rows, stride, a, grad, grad_stride, stream)
                : launch<T, false, false>(logits, rows, stride, a, grad, grad_stride, stream);
}

cudaError_t launch_distill_loss(const void *logits, int dtype, int rows, int vocab, int64_t stride,
                                const int32_t *labels, const int32_t *top_ids,
                                const float *top_logp, const float *log_rest, int k, float alpha,
                                float temperature, const float *row_weight, float *row_loss,
                                float *loss, void *grad, int64_t grad_stride, cudaStream_t stream) {
  const LossArgs a = {labels, top_ids, top_logp, log_rest, row_weight, row_loss,
                      vocab, k, alpha, temperature};
  cudaError_t err = dtype == SLIMWISE_DTYPE_BF16
                        ? launch<__nv_bfloat16>(logits, rows, stride, a, grad, grad_stride, stream)
                        : launch<float>(logits, rows, stride, a, grad, grad_stride, stream);
  if (err != cudaSuccess || !loss) return err;
  loss_sum_kernel<<<1, 1024, 0, stream>>>(row_loss, row_weight, rows, loss);
  return cudaGetLastError();
}

}  // namespace slimwise
