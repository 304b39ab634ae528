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
// elements out of the sums.  Where the list lies far above all of them, they keep
// a reference of their own, so that Q and the residual's share r q_i / Q hold
// however small Q is.
//
// A cluster handles a row.  For the gradient each CTA has its part copied into
// shared memory, in chunks that are all asked for at once, and sums exponentials
// against a running maximum as they come; for the loss alone the part passes
// through registers.  Each warp hands its sums to every CTA of the cluster, by
// stores that the receivers' mbarriers count (a cluster barrier would wait for
// the CTA's other memory operations too), each warp then joins all of them with
// the list by itself, and the gradient is computed from shared memory: one read
// and one write of the row, which bound the kernel.
//
// 4096 rows of 131072 bf16 with the gradient: 350 us, 5.8 TB/s (0.86 of a copy);
// 1021 rows of 65537 fp32 at a temperature 97 us, 5.3 TB/s, with two exponentials
// an element in each direction; the loss alone of 2048 rows of 150001 bf16 103 us,
// 5.4 TB/s.  What is left is the CTAs' turns: a part is read, summed, exchanged
// and written, and with three parts on an SM reads do not always overlap writes.
// 8 rows of 32000: 9 us replayed from a graph, two launches and their latency.
#include "vocab.cuh"

namespace slimwise {

constexpr int kLossThreads = 256;
constexpr int kLossWarps = kLossThreads / 32;
constexpr int kLossUnroll = 4;
constexpr int kChunk = kLossThreads * kLossUnroll;  // windows of a step, and of a copy (16 KB)
// CTAs of an SM, with and without gradient.  The loss alone of 2048 x 150001 bf16
// takes 8 us longer with four; at a temperature, where five spill 64 bytes a thread,
// it takes the same with both (147 to 149 us, around the whole call).
constexpr int kGradCtas = 4, kLossCtas = 5;
constexpr int kSliceMax = 200 * 1024;               // bytes of a row that one CTA may hold
constexpr int kAhead = 2;                            // steps that the loss alone prefetches
constexpr int kChunksMax = kSliceMax / (kChunk * 16) + 1;
static_assert(kTopMax <= kLossThreads, "one thread per list entry");
constexpr int kLossCluster = 16;                     // most CTAs of a row
// Bits of the exponent between the row's largest logit and the largest outside the
// list from which on those outside have a reference of their own: they then add next
// to nothing to the row's sum, and below it the largest of them is far from underflow.
constexpr float kFarBits = 40.0f;
constexpr int kLaneParts = kLossCluster * kLossWarps / 32;  // of the cluster's warps, a lane's

struct LossArgs {
  const int32_t *labels, *top_ids;
  const float *top_logp, *log_rest, *row_weight;
  float *row_loss;
  int vocab, K;
  float alpha, tau;
  bool summed;  // the kernel that sums the row losses follows
};

struct LossShared {
  int id[kTopMax];                        // the list: ids (-1: absent), logits, log P and P
  float z[kTopMax], lp[kTopMax], p[kTopMax];
  uint64_t bar[kChunksMax];
  uint64_t parts;                         // counts the bytes of the cluster's warps' sums
};

__device__ __forceinline__ float warp_max(float v) { return unordered(__reduce_max_sync(0xFFFFFFFFu, ordered(v))); }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
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
__device__ __forceinline__ uint4 packed(const float (&f)[16 / sizeof(T)]) {
  if constexpr (sizeof(T) == 4) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                      __float_as_uint(f[3]));
  } else {
    uint32_t u[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[q]) : "f"(f[2 * q + 1]), "f"(f[2 * q]));
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
}

template <typename T>
__device__ __forceinline__ void store_window(T *g, const Row<T> &row, int i,
                                             const float (&f)[Row<T>::E]) {
  constexpr int E = Row<T>::E;
  const int id0 = i * E - row.mis;
  if (row.whole(i)) {
    *reinterpret_cast<uint4 *>(g + id0) = packed<T>(f);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (id0 + e >= 0 && id0 + e < row.vocab) store(g + id0 + e, f[e]);
  }
}

// The 16 bytes that start `at` bytes into two neighbouring windows, 0 < at < 16
// and a multiple of the element's size; `at` is the same for all threads.
template <typename T>
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b, int at) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (at & 8)
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  if (at & 4)
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  if (sizeof(T) == 2 && at & 2)
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// kTemp: tau is not 1, so that p and q are two softmaxes.  kAlike: the gradient's
// rows are aligned as the logits' (the code for others costs 1% beside them).
template <typename T, bool kGrad, bool kTemp, bool kAlike>
__global__ void __launch_bounds__(kLossThreads, kGrad ? kGradCtas : kLossCtas)
    distill_loss_kernel(const T *logits, int64_t stride, LossArgs a, T *grad, int64_t grad_stride) {
  constexpr int E = Row<T>::E;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ LossShared sh;
  if (a.summed) pdl_launch_dependents();
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, V = a.vocab;
  const int64_t t = blockIdx.x / C;
  const int label = a.labels[t];
  const Row<T> row(logits + t * stride, V);
  const int per = (row.windows + C - 1) / C;
  const int lo = min(rank * per, row.windows), hi = min(lo + per, row.windows);
  const int id_lo = max(lo * E - row.mis, 0), id_hi = min(hi * E - row.mis, V);
  T *const g = kGrad ? grad + t * grad_stride : nullptr;
  // gradient rows that start like the logits' are written in the same windows
  const bool alike = kAlike || ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(row.p)) & 15) == 0;
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

  // a word of bits for each thread and step: 8 for each of its windows
  uint4 *const slice = reinterpret_cast<uint4 *>(smem);
  uint32_t *const bits = reinterpret_cast<uint32_t *>(smem + (kGrad ? (size_t)per * 16 : 0));
  // each warp's reference, sum for p, sum for q, of the cluster's warps
  float4 *const parts = reinterpret_cast<float4 *>(bits + (per + kChunk - 1) / kChunk * kLossThreads);
  const int chunks = (hi - lo + kChunk - 1) / kChunk;
  if (tid == 0) {
    mbar_init(smem_u32(&sh.parts), 1);
    if constexpr (kGrad)
      for (int i = 0; i < chunks; ++i) mbar_init(smem_u32(&sh.bar[i]), 1);
    mbar_fence_init();
    mbar_arrive_expect_tx(smem_u32(&sh.parts), (uint32_t)(C * kLossWarps * sizeof(float4)));
    if constexpr (kGrad)
      for (int i = 0; i < chunks; ++i) {
        // the row's partial windows at its ends are left out
        const int at = lo + i * kChunk, from = max(at, row.whole_lo);
        const int to = min(min(at + kChunk, hi), row.whole_lo + row.whole_n);
        const uint32_t bytes = to > from ? (uint32_t)(to - from) * 16 : 0;
        mbar_arrive_expect_tx(smem_u32(&sh.bar[i]), bytes);
        if (bytes) bulk_load(smem_u32(slice + (from - lo)), row.w + from, bytes, smem_u32(&sh.bar[i]));
      }
  }
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // its mbarrier can be used
  // the loss alone has the steps to come brought into L2
  auto prefetch = [&](int b) {
    const int from = max(lo + b * kChunk, row.whole_lo);
    const int to = min(min(lo + (b + 1) * kChunk, hi), row.whole_lo + row.whole_n);
    if (to > from) bulk_prefetch(row.w + from, (uint32_t)(to - from) * 16);
  };
  if (!kGrad && tid == 0)
    for (int b = 0; b < kAhead; ++b) prefetch(b);
  int id = -1;
  float lp = 0.0f;
  if (tid < a.K) {
    id = a.top_ids[t * a.K + tid];
    lp = a.top_logp[t * a.K + tid];
  }
  for (int i = 0; i < chunks; ++i) bits[i * kLossThreads + tid] = 0;
  if constexpr (kGrad)
    for (int i = tid; i < 2; i += kLossThreads) {
      const int at = i ? row.windows - 1 : 0;
      if (at >= lo && at < hi && !row.whole(at)) slice[at - lo] = load_window(row, at);
    }
  const bool bad = __syncthreads_or(id >= V) || label >= V;
  if (bad) id = -1;
  float z = -INFINITY, zy = 0.0f;
  if (id >= 0) z = to_float(row.p[id]);
  if (!bad) zy = to_float(row.p[label]);
  if (id >= id_lo && id < id_hi) {
    const int i = (id + row.mis) / E - lo;
    atomicOr(&bits[i / kChunk * kLossThreads + i % kLossThreads],
             1u << (i % kChunk / kLossThreads * 8 + (id + row.mis) % E));
  }
  __syncthreads();

  // sums of the exponentials outside the list, against the largest so far: s1
  // of 2^((z - ref) c1), and with a temperature s2 of 2^((z - ref) c2)
  const float c1 = kLog2e, c2 = kTemp ? kLog2e / a.tau : kLog2e;
  float s1 = 0.0f, s2 = 0.0f, ref = kFloorRef;
  bool came = true;
  for (int b = 0; b < chunks; ++b) {
    if constexpr (kGrad) came = came && wait_copy(smem_u32(&sh.bar[b]), 0);
    else if (tid == 0) prefetch(b + kAhead);
    const uint32_t mask = bits[b * kLossThreads + tid];
    const int i0 = b * kChunk + tid;
    uint4 v[kLossUnroll];
    if ((b + 1) * kChunk <= hi - lo) {
#pragma unroll
      for (int u = 0; u < kLossUnroll; ++u)
        v[u] = kGrad ? slice[i0 + u * kLossThreads] : load_window(row, lo + i0 + u * kLossThreads);
    } else {
#pragma unroll
      for (int u = 0; u < kLossUnroll; ++u) {
        const int i = i0 + u * kLossThreads;
        const uint32_t none = neg_inf_bits(row.p);
        v[u] = make_uint4(none, none, none, none);
        if (lo + i < hi) v[u] = kGrad ? slice[i] : load_window(row, lo + i);
      }
    }
    if (mask) {
#pragma unroll
      for (int u = 0; u < kLossUnroll; ++u) v[u] = without<T>(v[u], mask >> (8 * u) & 0xFFu);
    }
    const float n = fmaxf(ref, fmaxf(window_max<T, false>(v[0], v[1]), window_max<T, false>(v[2], v[3])));
    s1 = fmaf(s1, exp_from(ref, n, c1), windows_sum<T, kLossUnroll>(v, c1, n));
    if constexpr (kTemp) s2 = fmaf(s2, exp_from(ref, n, c2), windows_sum<T, kLossUnroll>(v, c2, n));
    ref = n;
  }
  if (!came) s1 = s2 = NAN;
  // over the warp, then to every CTA of the cluster
  {
    const float top = warp_max(ref);
    s1 = warp_sum(s1 * exp_from(ref, top, c1));
    if constexpr (kTemp) s2 = warp_sum(s2 * exp_from(ref, top, c2));
    ref = top;
  }
  if (tid < a.K) {
    sh.id[tid] = id;
    sh.z[tid] = z;
    sh.lp[tid] = lp;
    sh.p[tid] = id >= 0 ? expf(lp) : 0.0f;
  }
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  // (with zy, so that it has been read when another CTA may write over it in place;
  // the list's logits are in shared memory by now)
  if (lane < C) {
    const uint32_t to = mapa_shared(smem_u32(&parts[rank * kLossWarps + (tid >> 5)]), lane);
    asm volatile(
        "st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to),
        "f"(ref), "f"(s1), "f"(s2), "f"(zy), "r"(mapa_shared(smem_u32(&sh.parts), lane))
        : "memory");
  }
  __syncthreads();  // the list
  if (!mbar_wait_cluster_bounded(smem_u32(&sh.parts), 0, nullptr, kDefaultWaitLimitNs)) came = false;
  const bool lost = !__all_sync(0xFFFFFFFFu, came);

  // the row's sums, by each warp for itself: the parts, and the list
  float4 part[kLaneParts];
  float top = kFloorRef;
#pragma unroll
  for (int j = 0; j < kLaneParts; ++j) {
    const int i = lane + 32 * j;
    part[j] = make_float4(kFloorRef, 0.0f, 0.0f, 0.0f);
    if (i < C * kLossWarps) part[j] = parts[i];
    top = fmaxf(top, part[j].x);
  }
  const float rest_top = warp_max(top);
  for (int i = lane; i < a.K; i += 32) top = fmaxf(top, sh.z[i]);
  ref = warp_max(top);
  const float rest_ref = (ref - rest_top) * c2 > kFarBits ? rest_top : ref;
  float rest1 = 0.0f, rest2 = 0.0f;
#pragma unroll
  for (int j = 0; j < kLaneParts; ++j) {
    if (32 * j >= C * kLossWarps) break;
    rest1 += part[j].y * exp_from(part[j].x, rest_ref, c1);
    if constexpr (kTemp) rest2 += part[j].z * exp_from(part[j].x, rest_ref, c2);
  }
  rest1 = warp_sum(rest1);
  rest2 = kTemp ? warp_sum(rest2) : rest1;
  float list1 = 0.0f, list2 = 0.0f, M = 0.0f;
  bool y_listed = false;
  for (int i = lane; i < a.K; i += 32) {
    list1 += exp_from(sh.z[i], ref, c1);
    if constexpr (kTemp) list2 += exp_from(sh.z[i], ref, c2);
    M += sh.p[i];
    y_listed |= sh.id[i] == label;
  }
  y_listed = __any_sync(0xFFFFFFFFu, y_listed);
  const float lr = a.log_rest[t], r = expf(lr);
  // totals against ref: the elements outside the list count for scale1, scale2 (1
  // where their reference is the row's)
  const float scale1 = exp_from(rest_ref, ref, c1), scale2 = kTemp ? exp_from(rest_ref, ref, c2) : scale1;
  const float total1 = bad || lost ? NAN : fmaf(rest1, scale1, warp_sum(list1));
  const float total2 = kTemp ? (bad || lost ? NAN : fmaf(rest2, scale2, warp_sum(list2))) : total1;
  M = warp_sum(M) + r;
  const float w = a.row_weight ? a.row_weight[t] : 1.0f;
  const float beta = (1.0f - a.alpha) * a.tau;
  if (rank == 0 && tid < 32) {
    // CE and tau KL from differences of logits as they are: those from a logit of the
    // type's lowest value are finite, and not so times log2 e or over a small tau
    // (a target that is not a number is not 0: it makes the loss NaN, as the gradient)
    const float l1 = logf(total1), l2 = kTemp ? a.tau * logf(total2) : l1;
    float kl = 0.0f;
    for (int i = lane; i < a.K; i += 32) {
      const float P = sh.p[i];
      if (P != 0.0f) kl += P * (a.tau * sh.lp[i] + l2 - (sh.z[i] - ref));
    }
    kl = warp_sum(kl);
    if (lane == 0) {
      const float ce = l1 - (zy - ref);
      const float kr = r != 0.0f ? r * (a.tau * (lr - logf(rest2 / total2)) - (rest_ref - ref)) : 0.0f;
      // an infinite term without weight is 0, as it is in the gradient
      auto weighted = [](float by, float x) { return by == 0.0f && x == INFINITY ? 0.0f : by * x; };
      a.row_loss[t] = weighted(a.alpha, ce) + weighted(beta, kl + kr);
    }
  }
  if constexpr (kGrad) {
    // outside the list: A e1 + B e2, exponentials against rest_ref (B into A when
    // there is one softmax).  A listed element's may overflow; it is written again.
    const float share = rest2 > 0.0f ? r / rest2 : 0.0f;
    float A = w * a.alpha * scale1 / total1;
    float B = w * beta * (M * scale2 / total2 - share);
    if constexpr (!kTemp) A += B;
    auto outside = [&](float x) {
      float v = A * exp_from(x, rest_ref, c1);
      if constexpr (kTemp) v = fmaf(B, exp_from(x, rest_ref, c2), v);
      return v;
    };
    const uint64_t mr = pair(-rest_ref, -rest_ref), cc1 = pair(c1, c1), cc2 = pair(c2, c2);
    const uint64_t AA = pair(A, A), BB = pair(B, B);
    auto window = [&](uint4 v, auto put) {
      constexpr int P = E / 2;
      uint64_t p[P];
      unpack_pairs<T>(v, p);
      float f[E];
#pragma unroll
      for (int q = 0; q < P; ++q) {
        uint64_t v = mul2(AA, exp2_pair(p[q], mr, cc1));
        if constexpr (kTemp) v = add2(v, mul2(BB, exp2_pair(p[q], mr, cc2)));
        split(v, f[2 * q], f[2 * q + 1]);
      }
      put(f);
    };
    if (alike) {
      const int from = max(lo, row.whole_lo), to = min(hi, row.whole_lo + row.whole_n);
      uint4 *const gw = reinterpret_cast<uint4 *>(g - row.mis);
#pragma unroll 4
      for (int i = from + tid; i < to; i += kLossThreads)
        window(slice[i - lo], [&](const float (&f)[E]) { gw[i] = packed<T>(f); });
      // the row's partial windows
      for (int i = tid; i < 2; i += kLossThreads) {
        const int at = i ? row.windows - 1 : 0;
        if (at >= lo && at < hi && !row.whole(at))
          window(slice[at - lo], [&](const float (&f)[E]) { store_window(g, row, at, f); });
      }
    } else {
      // windows of the gradient, each from two of the logits', and the elements
      // before and after them (4096 rows of 131072 bf16: 373 us, an element at a
      // time 402; gradients of the same alignment 350)
      const int before = min((int)((16 - (reinterpret_cast<uintptr_t>(g + id_lo) & 15)) & 15) / (int)sizeof(T),
                             max(id_hi - id_lo, 0));
      const int from = id_lo + before, n = max(id_hi - from, 0) / E;
      const int first = from + row.mis - lo * E, at = first % E * (int)sizeof(T);
      const uint4 *const src = slice + first / E;
      uint4 *const gw = reinterpret_cast<uint4 *>(g + from);
#pragma unroll 2
      for (int i = tid; i < n; i += kLossThreads)
        window(shifted<T>(src[i], src[i + 1], at), [&](const float (&f)[E]) { gw[i] = packed<T>(f); });
      const T *const part = reinterpret_cast<const T *>(slice) + row.mis - lo * E;
      const int after = max(id_hi - from, 0) - n * E;
      if (tid < before) store(g + id_lo + tid, outside(to_float(part[id_lo + tid])));
      if (tid < after) store(g + from + n * E + tid, outside(to_float(part[from + n * E + tid])));
    }
    // then the list's elements and the label
    __syncthreads();
    if (!bad && id >= id_lo && id < id_hi) {
      const float on = id == label ? a.alpha : 0.0f;
      const float e1 = exp_from(z, ref, c1), e2 = kTemp ? exp_from(z, ref, c2) : e1;
      store(g + id, w * (a.alpha * (e1 / total1) - on + beta * (M * (e2 / total2) - sh.p[tid])));
    }
    if (!bad && tid == 0 && !y_listed && label >= id_lo && label < id_hi)
      store(g + label, outside(zy) - w * a.alpha);
    // a copy that did not come in time may still come: not after this CTA's end
    if (lost)
      for (int b = 0; b < chunks; ++b) wait_copy(smem_u32(&sh.bar[b]), 0);
  }
}

// loss = sum of weight x row loss over the rows with a label, whatever the others'
// weights (1 / the number of labelled rows may be 1 / 0): thread i adds its rows i,
// i + 1024, ... in order, in fp64, then a butterfly and the warps in turn: the same
// every time.
// (row_loss is still written when this kernel starts: no __restrict__)
__global__ void __launch_bounds__(1024)
    loss_sum_kernel(const float *row_loss, const int32_t *__restrict__ labels,
                    const float *__restrict__ row_weight, int rows, float *loss) {
  __shared__ double part[32];
  pdl_wait_primary();
  double s = 0.0;
  for (int t = threadIdx.x; t < rows; t += 1024) {
    const double l = (double)row_loss[t] * (row_weight ? (double)row_weight[t] : 1.0);
    s += labels[t] >= 0 ? l : 0.0;
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 32; ++w) s += part[w];
    *loss = (float)s;
  }
}

// Shared memory of a CTA that takes `per` windows, one of C of a row.
static size_t loss_smem(int per, int C, bool grad) {
  return (grad ? (size_t)per * 16 : 0) + (size_t)(per + kChunk - 1) / kChunk * kLossThreads * 4 +
         (size_t)C * kLossWarps * sizeof(float4);
}
// CTAs of a row.  With the gradient, the number that lets the CTAs of an SM hold
// the most of their rows at once: at 131072 bf16, parts of 65 KB three to an SM
// took 363 us for 4096 rows, 44 KB four 385, 33 KB five 392, 87 KB two 413.  One
// CTA alone on an SM does not read while it writes (380000 bf16, 512 rows: parts
// of 190 KB 179 us, of 95 KB 152), and two less than three (1000 rows of 128256
// fp32: 2 x 100 KB 177, 3 x 63 KB 168): they count for 9/10.  Each CTA also costs
// its row's exchange: the fewest that come within a few percent.
// Where few rows leave SMs idle, more.
static int loss_ctas(int rows, int windows, bool grad) {
  int best = 1;
  if (grad) {
    size_t most = 0;
    for (int C = 1; C <= kLossCluster; ++C) {
      const int per = (windows + C - 1) / C;
      if (per * 16 > kSliceMax) continue;
      const int ctas = (int)(228 * 1024 / (loss_smem(per, C, true) + sizeof(LossShared) + 1024));
      if (ctas < 2) continue;
      size_t held = (size_t)(ctas < kGradCtas ? ctas : kGradCtas) * per;
      if (ctas == 2) held -= held / 10;
      if (held > most + most / 32) {
        most = held;
        best = C;
      }
    }
  }
  // the loss alone: two for long rows (150001 bf16, 2048 rows: 101 us, with one 103, with three 109)
  if (!grad && windows >= 16 * kChunk) best = 2;
  while (best <= kClusterMax / 2 && rows * best <= 152 && windows >= 2 * best * kLossThreads) best *= 2;
  return best;
}

template <typename T, bool kGrad, bool kTemp, bool kAlike>
static cudaError_t launch(const void *logits, int rows, int64_t stride, const LossArgs &a,
                          void *grad, int64_t grad_stride, cudaStream_t stream) {
  constexpr int E = Row<T>::E;
  const int windows = (a.vocab + 2 * E - 2) / E;  // the most that a row can cover
  const int C = loss_ctas(rows, windows, kGrad);
  return launch_clusters<distill_loss_kernel<T, kGrad, kTemp, kAlike>, kGrad>(rows, C, kLossThreads,
                         loss_smem((windows + C - 1) / C, C, kGrad),
                         loss_smem(kSliceMax / 16, kLossCluster, true), stream, static_cast<const T *>(logits),
                         stride, a, static_cast<T *>(grad), grad_stride);
}

template <typename T>
static cudaError_t launch(const void *logits, int rows, int64_t stride, const LossArgs &a,
                          void *grad, int64_t grad_stride, cudaStream_t stream) {
  const bool temp = a.tau != 1.0f;
  if (!grad)
    return temp ? launch<T, false, true, true>(logits, rows, stride, a, grad, grad_stride, stream)
                : launch<T, false, false, true>(logits, rows, stride, a, grad, grad_stride, stream);
  const bool alike = (reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(grad)) % 16 == 0 &&
                     (stride - grad_stride) * (int64_t)sizeof(T) % 16 == 0;
  if (alike)
    return temp ? launch<T, true, true, true>(logits, rows, stride, a, grad, grad_stride, stream)
                : launch<T, true, false, true>(logits, rows, stride, a, grad, grad_stride, stream);
  return temp ? launch<T, true, true, false>(logits, rows, stride, a, grad, grad_stride, stream)
              : launch<T, true, false, false>(logits, rows, stride, a, grad, grad_stride, stream);
}

cudaError_t launch_distill_loss(const void *logits, int dtype, int rows, int vocab, int64_t stride,
                                const int32_t *labels, const int32_t *top_ids,
                                const float *top_logp, const float *log_rest, int k, float alpha,
                                float temperature, const float *row_weight, float *row_loss,
                                float *loss, void *grad, int64_t grad_stride, cudaStream_t stream) {
  const LossArgs a = {labels, top_ids, top_logp, log_rest, row_weight, row_loss,
                      vocab, k, alpha, temperature, loss != nullptr};
  cudaError_t err = dtype == SLIMWISE_DTYPE_BF16
                        ? launch<__nv_bfloat16>(logits, rows, stride, a, grad, grad_stride, stream)
                        : launch<float>(logits, rows, stride, a, grad, grad_stride, stream);
  if (err != cudaSuccess || !loss) return err;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1);
  cfg.blockDim = dim3(1024);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, loss_sum_kernel, (const float *)row_loss, labels, row_weight, rows, loss);
}

}  // namespace slimwise
