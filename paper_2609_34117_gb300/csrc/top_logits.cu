// top_logits.cu -- a teacher's targets for distillation: the K largest logits
// of each row as log-probabilities, and the log of the mass that the others
// hold (SlimWise Sec. 3.3, Eq. 3: top-K of the teacher plus a residual bucket).
//
//   S    = ids of the K largest z (larger value first, then the lower id)
//   logp = z_S / tau - log sum_i exp(z_i / tau)
//   log_rest = log (sum_{i not in S} exp(z_i / tau)) - log sum_i exp(z_i / tau)
//
// The mass of the others is summed over them, not taken as 1 - the list's: a
// teacher that is nearly sure leaves 1e-6, which the difference would not hold.
//
// One read of the logits (vocab.cuh has the scan), a few hundred bytes written a
// row.  4096 rows of 131072 bf16, K = 64: 223 us, 4.8 TB/s (0.71 of a copy), with
// the schedulers issuing in 79 % of the cycles: bound by its instructions, 12.5 a
// warp and 32 elements, of which a step's exponentials and sums are 3.6 and the
// rest the maxima, copies, lists, thresholds and a row's end.  511 rows of 150001
// fp32: 70 us, 4.3 TB/s; 511 rows on 152 SMs leave some with four and some with
// three, which alone takes 54.  One row of 131072 bf16: 13 us, one after the other a
// launch, 8 CTAs' scan and the leader's join (their shares are not measured).  Above K = 64 a kernel of its own
// holds long lists and candidates, and leaves room for three CTAs on an SM: 4096
// rows of 131072 bf16 at K = 100 281 us, at K = 256 428 (selecting and ranking 256
// of about 450 candidates a row); 1181 of 22705 bf16 at K = 256 89 us.
#include "vocab.cuh"

namespace slimwise {

// Stages of the rings where the rows are few: 152 rows of 150001 fp32 take 23.5 us
// with three and 26.3 with two, 304 of 131072 bf16 24.6 and 26.5, 16 rows in
// clusters 17.0 and 18.1.
constexpr int kFewStages = 3;
__host__ __device__ constexpr int top_stages(int ctas) { return ctas == kFewCtas ? kFewStages : kManyStages; }

template <typename T, bool kCluster, bool kLong, int kCtas>
__global__ void __launch_bounds__(kScanThreads, kCtas)
    top_logits_kernel(const T *__restrict__ logits, int64_t stride, int rows, int vocab, int K,
                      float c, float inv, int32_t *__restrict__ ids, float *__restrict__ logp,
                      float *__restrict__ log_rest) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int kStages = top_stages(kCtas);
  auto &sh = *reinterpret_cast<ScanShared<kStages> *>(smem);
  const int tid = threadIdx.x;
  Scan<T, kCluster, false, kLong, kStages> scan(sh, list_room(K), K, logits, stride, vocab, rows);
  auto request = [&](int, int &k, float &cc, bool &sums) {
    k = K;
    cc = c;
    sums = true;
  };
  scan.rows_of_cluster(request, [&](int t, int n) {
    // a candidate's place in the order, by a few lanes
    const int lanes = candidate_lanes(n), at_cand = tid / lanes, sub = tid % lanes;
    uint64_t key = at_cand < n ? sh.cand[at_cand] : 0;
    int rank = 0;
    if (key) {
#pragma unroll 4
      for (int i = sub; i < n; i += lanes) rank += sh.cand[i] > key;
    }
    for (int o = 1; o < lanes; o *= 2) rank += __shfl_xor_sync(0xFFFFFFFFu, rank, o);
    if (sub) key = 0;
    if (key) sh.by_rank[rank] = key_value(key);
    __syncthreads();
    // sums in the order of the ranks
    const float m = fmaxf(n > 0 ? sh.by_rank[0] : -INFINITY, kFloorRef);
    // the rest relative to the last of the list, which it does not exceed
    const float last = n >= K ? fmaxf(sh.by_rank[K - 1], kFloorRef) : scan.ref;
    float rest = scan.s * exp_from(scan.ref, last, c), e = 0.0f;
    if (tid < n) {
      if (tid < K) e = exp_from(sh.by_rank[tid], m, c);
      else rest += exp_from(sh.by_rank[tid], last, c);
    }
    const float scale = (last - m) * inv;  // log of the rest's scale
    rest = block_reduce<kScanThreads>(rest, sh.redf, OpAdd());
    const float top = block_reduce<kScanThreads>(e, sh.redf, OpAdd());
    const float mass = rest * expf(scale), total = mass + top, log_total = logf(total);
    const int64_t at = (int64_t)t * K;
    if (key && rank < K) {
      ids[at + rank] = (int32_t)key_index(key);
      logp[at + rank] = (key_value(key) - m) * inv - log_total;
    }
    // a row with NaN can have fewer candidates than K
    if (tid >= n && tid < K) {
      ids[at + tid] = -1;
      logp[at + tid] = NAN;
    }
    // of the rest's share, not a difference of two logarithms, which cancels where
    // the rest is most of the row; but so where the rest's mass underflows
    if (tid == 0)
      log_rest[t] = mass >= top        ? -log1pf(__fdividef(top, mass))
                    : mass > 0x1p-60f ? logf(__fdividef(mass, total))
                                      : logf(rest) + scale - log_total;
  });
}

ScanGrid scan_grid(int rows, int vocab, int element_bytes, int room, int K, bool long_lists, int few_stages,
                   size_t more_smem) {
  const int windows = (int)(((int64_t)vocab * element_bytes + 15) / 16) + 1;
  int C = 1;
  while (C < kClusterMax && rows * C <= 128 && windows >= 2 * C * 2 * kScanWarps * kWarpStep) C *= 2;
  const auto with = [&](int ctas) {
    const int stages = ctas == kFewCtas ? few_stages : kManyStages;
    const size_t smem = scan_smem(stages, room, K, C, long_lists) + more_smem;
    const int fit = (int)(228 * 1024 / (smem + 1024)), at_once = 152 * (fit < ctas ? fit : ctas) / C;
    return ScanGrid{C, rows < at_once ? rows : at_once, ctas == kFewCtas, smem};
  };
  const ScanGrid few = with(kFewCtas);
  return few.clusters == rows || C > 1 ? few : with(kManyCtas);
}

template <typename T, bool kCluster, bool kLong, int kCtas>
static cudaError_t launch_top(const ScanGrid &g, const void *logits, int rows, int vocab, int64_t stride,
                              int k, float temperature, int32_t *ids, float *logp, float *log_rest,
                              cudaStream_t stream) {
  const int most = kLong ? kTopMax : 64;
  return launch_clusters<top_logits_kernel<T, kCluster, kLong, kCtas>>(
      g.clusters, g.C, kScanThreads, g.smem,
      scan_smem(top_stages(kCtas), list_room(most), most, kCluster ? kClusterMax : 1, kLong), stream,
      static_cast<const T *>(logits), stride, rows, vocab, k, kLog2e / temperature, 1.0f / temperature, ids, logp, log_rest);
}
template <typename T, bool kLong>
static cudaError_t launch_top(const void *logits, int rows, int vocab, int64_t stride, int k,
                              float temperature, int32_t *ids, float *logp, float *log_rest,
                              cudaStream_t stream) {
  const ScanGrid g = scan_grid(rows, vocab, (int)sizeof(T), list_room(k), k, kLong, kFewStages, 0);
  const auto launch = g.C > 1 ? launch_top<T, true, kLong, kFewCtas>
                      : g.few ? launch_top<T, false, kLong, kFewCtas>
                              : launch_top<T, false, kLong, kManyCtas>;
  return launch(g, logits, rows, vocab, stride, k, temperature, ids, logp, log_rest, stream);
}
template <typename T>
static cudaError_t launch_top(const void *logits, int rows, int vocab, int64_t stride, int k,
                              float temperature, int32_t *ids, float *logp, float *log_rest,
                              cudaStream_t stream) {
  return k > 64 ? launch_top<T, true>(logits, rows, vocab, stride, k, temperature, ids, logp, log_rest, stream)
                : launch_top<T, false>(logits, rows, vocab, stride, k, temperature, ids, logp, log_rest, stream);
}

cudaError_t launch_top_logits(const void *logits, int dtype, int rows, int vocab, int64_t stride,
                              int k, float temperature, int32_t *ids, float *logp, float *log_rest,
                              cudaStream_t stream) {
  return dtype == SLIMWISE_DTYPE_BF16
             ? launch_top<__nv_bfloat16>(logits, rows, vocab, stride, k, temperature, ids, logp,
                                         log_rest, stream)
             : launch_top<float>(logits, rows, vocab, stride, k, temperature, ids, logp, log_rest,
                                 stream);
}

}  // namespace slimwise
