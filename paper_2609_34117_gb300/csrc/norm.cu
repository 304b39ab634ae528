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
// its CTA, so dg and db stay in its registers (many columns of a thread: in its shared
// memory) until the CTA's last row; a second kernel adds the CTAs' sums in order.
#include <type_traits>

#include "train.cuh"

namespace slimwise {

namespace {

// Sums of K values over a group of TPR threads, known to all of them.  `buf`: of
// the group, two sets of K values a warp, used in turn (`turn`), so that one
// barrier a reduction is enough.
template <int TPR, int K>
__device__ __forceinline__ void group_sum(float (&v)[K], float *buf, int &turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = warp_sum(v[k]);
  if constexpr (TPR > 32) {
    constexpr int W = TPR / 32;
    float *set = buf + turn * K * W;
    turn ^= 1;
    const int warp = threadIdx.x % TPR / 32, lane = threadIdx.x & 31;
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) set[k * W + warp] = v[k];
    asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / TPR), "n"(TPR) : "memory");
    // (the W sums of a value by W lanes, the same way in every warp)
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = set[k * W + (lane & (W - 1))];
#pragma unroll
      for (int o = W / 2; o >= 1; o >>= 1) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    }
  }
}

// How bf16 rows lie: on 16-byte boundaries and a multiple of 16 bytes long; anywhere; or
// anywhere, but a call's tensors alike, a row's start as far behind a boundary in each.
// (fp32 rows: 16 bytes an access, or an element, which costs them little.)
enum Form { kAligned, kAnywhere, kAlike };
// Rows that are not aligned: every eighth starts at the same distance from a boundary, so a
// CTA takes the rows of one class, r = class + 8 k.  Of such a row of the output, `body`
// elements behind the first `head` are whole windows; those before and behind it, 14 at
// the most, are held by the first threads of a group, one more element each (column `own`,
// else -1).  kAlike: the inputs' windows are the same, nothing is shifted.  kAnywhere:
// each access reads the two windows that its elements lie in, and shifts them.
constexpr int kClasses = 8;
template <bool kSame>
struct RowsOf {
  int cls, units, ctas, cta;  // rows of the class, and CTAs; this one
  int head, body, ends, own;
  // (t: of a group's threads; base: of a tensor with rows of `size` bytes an element)
  __device__ __forceinline__ RowsOf(int rows, int hidden, const void *base, int64_t stride, int size, int t) {
    cls = kSame ? (int)blockIdx.x % kClasses : 0;
    units = kSame ? (rows - cls + kClasses - 1) / kClasses : rows;
    ctas = kSame ? ((int)gridDim.x - cls + kClasses - 1) / kClasses : (int)gridDim.x;
    cta = kSame ? (int)blockIdx.x / kClasses : (int)blockIdx.x;
    const int v = 16 / size;
    const uintptr_t start = reinterpret_cast<uintptr_t>(base) + (uintptr_t)(cls * stride * size);
    head = kSame ? min((int)(-start & 15) / size, hidden) : 0;
    body = kSame ? (hidden - head) / v * v : hidden;
    ends = hidden - body;
    own = !kSame || t >= ends ? -1 : t < head ? t : body + t;
  }
  __device__ __forceinline__ int64_t row(int64_t unit) const { return kSame ? cls + kClasses * unit : unit; }
};
// Element `own` of a row, or 0, as it lies (bf16).
template <typename T>
__device__ __forceinline__ uint32_t read_own(const T *row, int own) {
  return own >= 0 ? (uint32_t)__ldg(reinterpret_cast<const unsigned short *>(row + own)) : 0u;
}
__device__ __forceinline__ float own_value(uint32_t bits) { return __uint_as_float(bits << 16); }
template <typename T>
__device__ __forceinline__ void write_own(T *row, int own, float v) {
  if (own >= 0) *reinterpret_cast<unsigned short *>(row + own) = (unsigned short)pack_bf16(v, 0.0f);
}

struct NormArgs {
  int rows, hidden;
  Extent x;
  int64_t stride, y_stride;
  const float *weight, *bias;
  float eps;
  float *mean, *rstd;
};

// Threads of a row (TPR) and elements of a thread (N): rows up to 256 (32, 8), 512,
// 1024, .. 8192 (32 .. 512, 16), 12288 (512, 24) and 16384 (512, 32).  Groups are persistent:
// the weight and bias of a thread's columns stay in its registers (24 and 32 elements: in
// shared memory; 2000 x 16000 bf16 35 us, read from the caches for each row 94), and R
// rows are on their way while R others are worked on.  Bound by memory and instructions:
// 16384 x 2048 bf16 layer norm 26 us, by itself 23 (a copy of as many bytes 23); with 8
// elements a thread 30, a row's sums costing as much as its elements.  bf16 rows of 4001,
// 32768 of them: alike in x and y 98 us, anywhere 133 (written through
// shared memory as whole windows 182, by element 230).
constexpr int kNormThreads = 256;
template <int TPR>
constexpr int kNormBlock = TPR > kNormThreads ? TPR : kNormThreads;
// (two fp32 rows of 16 in place of one: 8192 x 8192 92 -> 90 us, 32768 x 1000 49 -> 47)
template <bool kAny, int N>
constexpr int kNormRows = !kAny && N <= 16 ? 2 : 1;

template <typename T, int V, Form kForm, int TPR, int N, bool kLayer>
__global__ void __launch_bounds__(kNormBlock<TPR>, 512 / kNormBlock<TPR>)
    norm_kernel(const T *__restrict__ x, NormArgs a, T *__restrict__ y) {
  constexpr bool kAny = kForm == kAnywhere, kSame = kForm != kAligned;
  constexpr int R = kNormRows<kAny, N>, P = N / V, W = TPR / 32, kGroups = kNormBlock<TPR> / TPR;
  constexpr bool kHeld = N <= 16;
  using Part = RowPart<T, V, N>;
  __shared__ float2 buf[TPR > 32 ? 2 * R * kNormBlock<TPR> / 32 : 1];
  const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const float inv = 1.0f / (float)a.hidden;
  const RowsOf<kSame> rows(a.rows, a.hidden, y, a.y_stride, (int)sizeof(T), t);
  // columns of this warp, and of the warp whose sums this lane joins
  auto columns = [&](int warp) {
    int n = 0;
#pragma unroll
    for (int k = 0; k < P; ++k) n += max(0, min(rows.body - (k * TPR + 32 * warp) * V, 32 * V));
    return (float)(n + (warp == 0 ? rows.ends : 0));
  };
  const float warp_n = columns(t / 32), lane_n = columns(t & (W - 1));
  const float warp_inv = warp_n > 0.0f ? 1.0f / warp_n : 0.0f, lane_inv = lane_n > 0.0f ? 1.0f / lane_n : 0.0f;
  auto pair = [&](const float *p, int e) {
    const int c = Part::column(e, t, TPR), c1 = Part::column(e + 1, t, TPR);
    return f2(p && c < rows.body ? __ldg(p + rows.head + c) : 0.0f, p && c1 < rows.body ? __ldg(p + rows.head + c1) : 0.0f);
  };
  const float own_g = kSame && rows.own >= 0 ? __ldg(a.weight + rows.own) : 0.0f;
  const float own_o = kSame && rows.own >= 0 && a.bias ? __ldg(a.bias + rows.own) : 0.0f;
  // (32 elements a thread: in shared memory, [N / 2][TPR] of the weight, then of the bias)
  F2 g[kHeld ? N / 2 : 1], o[kHeld ? N / 2 : 1];
  extern __shared__ __align__(16) float held[];
  F2 *stored = reinterpret_cast<F2 *>(held) + t;
#pragma unroll
  for (int e = 0; e < N; e += 2) {
    (kHeld ? g[kHeld ? e / 2 : 0] : stored[e / 2 * TPR]) = pair(a.weight, e);
    (kHeld ? o[kHeld ? e / 2 : 0] : stored[(N / 2 + e / 2) * TPR]) = pair(a.bias, e);
  }
  using Coming = typename std::conditional<kAny, Windows<T, kAny ? N : 16 / sizeof(T)>, Part>::type;
  uint32_t own[R], own_next[R];  // kAlike: this thread's element beside the body
  auto fetch = [&](Coming (&p)[R], int64_t r0) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const T *row = x + (r0 + i < rows.units ? rows.row(r0 + i) : 0) * a.stride;
      const int width = r0 + i < rows.units ? rows.body : 0;
      if constexpr (kAny) p[i].load(row + rows.head, t, TPR, width, a.x);
      else p[i].load(row + rows.head, t, TPR, width);
      if (kSame && t < 32) own_next[i] = read_own(row, rows.own);
    }
  };
  auto arrive = [&](Part (&p)[R], const Coming (&next)[R]) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if constexpr (kAny) p[i].take(next[i], t, TPR, rows.body);
      else p[i] = next[i];
      if constexpr (kSame) own[i] = own_next[i];
    }
  };
  const int64_t step = (int64_t)rows.ctas * kGroups * R;
  int64_t r0 = ((int64_t)rows.cta * kGroups + group) * R;
  int turn = 0;
  Part p[R];
  Coming next[R];
  if (r0 < rows.units) {
    fetch(next, r0);
    arrive(p, next);
  }
  for (; r0 < rows.units; r0 += step) {
    fetch(next, r0 + step);
    float mu[R], q[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      mu[i] = 0.0f;
      if constexpr (kLayer) {
        F2 s = f2(0.0f);
#pragma unroll
        for (int e = 0; e < N; e += 2) s = add2(s, p[i].get2(e));
        const float2 h = halves(s);
        mu[i] = h.x + h.y;
        if (kSame && t < 32) mu[i] += own_value(own[i]);
        mu[i] = warp_sum(mu[i]);
      }
    }
    // the squares (layer norm: about the mean of the warp's columns)
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const F2 m = f2(-mu[i] * warp_inv);
      F2 s = f2(0.0f);
      // (not the row's width: of rows that start anywhere the ends are no columns of the threads)
      const bool full = rows.body == TPR * N;
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        F2 d = p[i].get2(e);
        if constexpr (kLayer) {
          d = add2(d, m);
          // (the last pieces may have columns past the row)
          if (!full && ((e + 1) / V + 1) * TPR * V > rows.body) {
            const float2 h = halves(d);
            d = f2(Part::column(e, t, TPR) < rows.body ? h.x : 0.0f, Part::column(e + 1, t, TPR) < rows.body ? h.y : 0.0f);
          }
        }
        s = fma2(d, d, s);
      }
      const float2 h = halves(s);
      q[i] = h.x + h.y;
      if (kSame && t < 32) {
        const float d = rows.own >= 0 ? own_value(own[i]) - (kLayer ? mu[i] * warp_inv : 0.0f) : 0.0f;
        q[i] = fmaf(d, d, q[i]);
      }
      q[i] = warp_sum(q[i]);
    }
    if constexpr (TPR > 32) {
      // of the row, a lane a warp: the warps' squares about their means, moved to the row's
      // mean; two sets in turn, so that one barrier is enough
      float2 *set = buf + (group * 2 + turn) * R * W;
      turn ^= 1;
      if ((t & 31) == 0)
#pragma unroll
        for (int i = 0; i < R; ++i) set[i * W + t / 32] = make_float2(mu[i], q[i]);
      asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(TPR) : "memory");
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float2 v = set[i * W + (t & (W - 1))];
        q[i] = v.y;
        if constexpr (kLayer) {
          mu[i] = v.x;
#pragma unroll
          for (int k = W / 2; k >= 1; k >>= 1) mu[i] += __shfl_xor_sync(0xFFFFFFFFu, mu[i], k);
          mu[i] *= inv;
          const float d = fmaf(v.x, lane_inv, -mu[i]);
          q[i] = fmaf(lane_n * d, d, q[i]);
        }
#pragma unroll
        for (int k = W / 2; k >= 1; k >>= 1) q[i] += __shfl_xor_sync(0xFFFFFFFFu, q[i], k);
      }
    } else if constexpr (kLayer) {
#pragma unroll
      for (int i = 0; i < R; ++i) mu[i] *= inv;
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (r0 + i >= rows.units) continue;
      const int64_t r = rows.row(r0 + i);
      const float rs = rsqrtf(fmaf(q[i], inv, a.eps));
      if (t == 0) {
        a.rstd[r] = rs;
        if constexpr (kLayer) a.mean[r] = mu[i];
      }
      const F2 m = f2(-mu[i]), f = f2(rs);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        F2 v = p[i].get2(e);
        if constexpr (kLayer) v = add2(v, m);
        if constexpr (kHeld) p[i].set2(e, fma2(mul2(v, f), g[e / 2], o[e / 2]));
        else p[i].set2(e, fma2(mul2(v, f), stored[e / 2 * TPR], stored[(N / 2 + e / 2) * TPR]));
      }
      p[i].store(y + r * a.y_stride + rows.head, t, TPR, rows.body);
      if (kSame && t < 32)
        write_own(y + r * a.y_stride, rows.own, fmaf((own_value(own[i]) - (kLayer ? mu[i] : 0.0f)) * rs, own_g, own_o));
    }
    arrive(p, next);
  }
}

struct GradArgs {
  int rows, hidden;
  Extent dy, x;
  int64_t dy_stride, stride, dx_stride;
  const float *weight, *mean, *rstd;
  float *partial;  // [CTAs][kLayer ? 2 : 1][hidden]
};

// Threads of a row (TPR) and elements of a thread (N): bf16 rows up to 256 (32, 8), 512
// (32, 16), 1024 (128, 8), 2048 (256, 8), 4096 (256, 16), 8192 (512, 16), 12288 (512, 24)
// and 16384 (512, 32); fp32 with more threads between, and 12 elements up to 6144 (10 up to
// 5120 take as long: 4099 x 5001 55.4 us with either, 20000 x 5001 214 against 212.6 with
// 12, behind a cold cache).  512 threads are on an SM, several groups to a CTA, whose sums
// are joined before they leave: as many CTAs as groups cost 4 us at 32768 x 1000.  Bound by
// memory and a row's barrier: 16384 x 2048 bf16 RMS norm 33 us by itself, 6.1 TB/s.  A ring
// of asynchronous copies in place of the next row in registers took 133 us for 6000 x 7168
// fp32, this 96.  bf16 rows of 4001, 32768 of them: alike in all tensors 162, anywhere 258.
template <int TPR>
constexpr int kBlock = TPR == 32 ? 256 : 512;
// Rows of a group at once; the next ones come into registers meanwhile where these hold
// both.  Of 8 elements a thread three bf16 rows where they are aligned (16384 x 2048 41.0 -> 37.9
// us, four spill), else two (fp32 8192 x 4096 82 -> 71); of more, one.
template <typename T, Form kForm, int N>
constexpr int kBatch = N != 8 ? 1 : sizeof(T) == 2 && kForm == kAligned ? 3 : 2;
// What of a thread does not stay in registers: the next row where it would take 64 of them
// (windows take twice as many on their way); the columns' sums where these, the rows and
// the next ones take 96 and more (aligned rows alone have room for 96); the weights of 24 columns
// and more (of fewer where the rows' ends are held besides: with windows, or 16 of layer norm).
// Sums and weights are then in shared memory.
template <typename T, Form kForm, int N>
constexpr bool kAhead = N * (int)sizeof(T) <= (kForm == kAnywhere ? 48 : 96);
template <typename T, Form kForm, int N, bool kLayer>
constexpr bool kSumsShared = (kLayer ? 2 : 1) * N + N * (int)sizeof(T) / 2 *
                             (1 + (kAhead<T, kForm, N> ? kForm == kAnywhere ? 2 : 1 : 0)) > (kForm == kAligned ? 96 : 95);
template <Form kForm, int N, bool kLayer>
constexpr bool kWeightsShared = N >= 24 || kForm == kAnywhere || (kForm == kAlike && kLayer && N == 16);

template <typename T, int V, Form kForm, int TPR, int N, bool kLayer>
__global__ void __launch_bounds__(kBlock<TPR>, 512 / kBlock<TPR>)
    norm_grad_kernel(const T *__restrict__ dy, const T *__restrict__ x, GradArgs a,
                     T *__restrict__ dx) {
  constexpr bool kAny = kForm == kAnywhere, kSame = kForm != kAligned;
  constexpr int R = kBatch<T, kForm, N>, K = kLayer ? 2 * R : R;
  constexpr int kGroups = kBlock<TPR> / TPR;
  constexpr bool kStored = kWeightsShared<kForm, N, kLayer>, kShared = kSumsShared<T, kForm, N, kLayer>;
  constexpr bool kNext = kAhead<T, kForm, N>;
  using Part = RowPart<T, V, N>;
  using Coming = typename std::conditional<kAny, Windows<T, kAny ? N : 16 / sizeof(T)>, Part>::type;
  struct Batch {
    Part d[R], x[R];
    float mu[R], rs[R];
  };
  struct ComingBatch {
    Coming d[R], x[R];
    float mu[R], rs[R];
  };
  __shared__ float buf[kGroups][2 * K * (TPR / 32)];
  // kShared: dg [N][TPR], db [N][TPR]; groups of a warp: one group's sums; kStored: weights [N][TPR]
  extern __shared__ __align__(16) float held[];
  int turn = 0;
  const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const float inv = 1.0f / (float)a.hidden;
  const RowsOf<kSame> rows(a.rows, a.hidden, dx, a.dx_stride, (int)sizeof(T), t);
  auto read_weight = [&](int e) {
    const int c = Part::column(e, t, TPR), c1 = Part::column(e + 1, t, TPR);
    return f2(c < rows.body ? __ldg(a.weight + rows.head + c) : 0.0f,
              c1 < rows.body ? __ldg(a.weight + rows.head + c1) : 0.0f);
  };
  // kAlike: this thread's element beside the body, of x and above it of dy
  uint32_t own[R], own_next[R];
  const float own_g = kSame && rows.own >= 0 ? __ldg(a.weight + rows.own) : 0.0f;
  float own_dg = 0.0f, own_db = 0.0f;
  auto own_x = [](uint32_t v) { return own_value(v); };
  auto own_dy = [](uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); };
  F2 *weights = reinterpret_cast<F2 *>(held) + (kShared || kGroups > 1 ? (kLayer ? 2 : 1) * (N / 2) * TPR : 0);
  F2 g[kStored ? 1 : N / 2], dg[kShared ? 1 : N / 2], db[kShared ? 1 : N / 2];
#pragma unroll
  for (int e = 0; e < N / 2; ++e) {
    if constexpr (kStored) weights[e * TPR + t] = read_weight(2 * e);
    else g[e] = read_weight(2 * e);
    if constexpr (kShared) {
      reinterpret_cast<F2 *>(held)[e * TPR + t] = f2(0.0f);
      if constexpr (kLayer) reinterpret_cast<F2 *>(held)[(N / 2 + e) * TPR + t] = f2(0.0f);
    } else {
      dg[e] = db[e] = f2(0.0f);
    }
  }
  auto weight = [&](int e) {
    if constexpr (kStored) return weights[e / 2 * TPR + t];
    else return g[e / 2];
  };
  auto fetch = [&](ComingBatch &b, int r0) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const bool in = r0 + i < rows.units;
      const int64_t r = in ? rows.row(r0 + i) : 0;
      if constexpr (kAny) {
        b.d[i].load(dy + r * a.dy_stride + rows.head, t, TPR, in ? rows.body : 0, a.dy);
        b.x[i].load(x + r * a.stride + rows.head, t, TPR, in ? rows.body : 0, a.x);
      } else {
        b.d[i].load(dy + r * a.dy_stride + rows.head, t, TPR, in ? rows.body : 0);
        b.x[i].load(x + r * a.stride + rows.head, t, TPR, in ? rows.body : 0);
      }
      if constexpr (kSame)
        own_next[i] = read_own(x + r * a.stride, in ? rows.own : -1) | read_own(dy + r * a.dy_stride, in ? rows.own : -1) << 16;
      b.rs[i] = in ? __ldg(a.rstd + r) : 0.0f;
      b.mu[i] = kLayer && in ? __ldg(a.mean + r) : 0.0f;
    }
  };
  const int step = rows.ctas * kGroups * R;
  int r0 = (rows.cta * kGroups + group) * R;
  Batch now;
  ComingBatch next;
  auto arrive = [&]() {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if constexpr (kAny) {
        now.d[i].take(next.d[i], t, TPR, rows.body);
        now.x[i].take(next.x[i], t, TPR, rows.body);
      } else {
        now.d[i] = next.d[i];
        now.x[i] = next.x[i];
      }
      if constexpr (kSame) own[i] = own_next[i];
      now.mu[i] = next.mu[i];
      now.rs[i] = next.rs[i];
    }
  };
  if (kNext && r0 < rows.units) {
    fetch(next, r0);
    arrive();
  }
  for (; r0 < rows.units; r0 += step) {
    fetch(next, !kNext ? r0 : r0 + step < rows.units ? r0 + step : rows.units);
    if constexpr (!kNext) arrive();
    float s[K];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const F2 u = f2(-now.mu[i]), v = f2(now.rs[i]);
      F2 sum = f2(0.0f), sum0 = f2(0.0f);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        // (columns past the row: dy = 0 and the weight 0)
        F2 n = now.x[i].get2(e);
        if constexpr (kLayer) n = add2(n, u);
        n = mul2(n, v);
        const F2 de = now.d[i].get2(e), ge = mul2(de, weight(e));
        sum = fma2(n, ge, sum);
        if constexpr (kLayer) sum0 = add2(sum0, ge);
        if constexpr (kShared) {
          F2 *at = reinterpret_cast<F2 *>(held) + (e / 2) * TPR + t;
          *at = fma2(de, n, *at);
          if constexpr (kLayer) at[N / 2 * TPR] = add2(at[N / 2 * TPR], de);
        } else {
          dg[e / 2] = fma2(de, n, dg[e / 2]);
          if constexpr (kLayer) db[e / 2] = add2(db[e / 2], de);
        }
      }
      const float2 h = halves(sum), h0 = halves(sum0);
      s[i] = h.x + h.y;
      if constexpr (kLayer) s[R + i] = h0.x + h0.y;
      if (kSame && t < 32) {
        const float n = (own_x(own[i]) - now.mu[i]) * now.rs[i], d = own_dy(own[i]);
        s[i] = fmaf(n, d * own_g, s[i]);
        own_dg = fmaf(d, n, own_dg);
        if constexpr (kLayer) {
          s[R + i] += d * own_g;
          own_db += d;
        }
      }
    }
    group_sum<TPR>(s, buf[group], turn);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (r0 + i >= rows.units) continue;
      // dx = rs g - rs m0 - n rs m
      const float rs = now.rs[i];
      const F2 u = f2(-now.mu[i]), v = f2(rs), m = f2(-rs * (s[i] * inv)), m0 = f2(kLayer ? -rs * (s[R + i] * inv) : 0.0f);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        F2 n = now.x[i].get2(e), ge = mul2(now.d[i].get2(e), weight(e));
        if constexpr (kLayer) n = add2(n, u);
        n = mul2(n, v);
        ge = kLayer ? fma2(ge, v, m0) : mul2(ge, v);
        now.x[i].set2(e, fma2(n, m, ge));
      }
      now.x[i].store(dx + rows.row(r0 + i) * a.dx_stride + rows.head, t, TPR, rows.body);
      if (kSame && t < 32) {
        const float n = (own_x(own[i]) - now.mu[i]) * rs, k = -rs * (s[i] * inv), k0 = kLayer ? -rs * (s[R + i] * inv) : 0.0f;
        write_own(dx + rows.row(r0 + i) * a.dx_stride, rows.own, fmaf(n, k, fmaf(own_dy(own[i]) * own_g, rs, k0)));
      }
    }
    if constexpr (kNext) arrive();
  }
  pdl_launch_dependents();
  // the CTA's sums: its groups' in turn
  float *out = a.partial + (int64_t)blockIdx.x * (kLayer ? 2 : 1) * a.hidden;
  F2 *mine = reinterpret_cast<F2 *>(held);
  if constexpr (kGroups > 1) {
    __shared__ float2 own_sum[kSame ? TPR : 1];
    for (int k = 0; k < kGroups; ++k) {
      if (group == k) {
        if constexpr (kSame) {
          if (k) {
            own_dg += own_sum[t].x;
            own_db += own_sum[t].y;
          }
          own_sum[t] = make_float2(own_dg, own_db);
        }
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          mine[e * TPR + t] = k ? add2(mine[e * TPR + t], dg[e]) : dg[e];
          if constexpr (kLayer) mine[(N / 2 + e) * TPR + t] = k ? add2(mine[(N / 2 + e) * TPR + t], db[e]) : db[e];
        }
      }
      __syncthreads();
    }
    if (group != 0) return;
    if constexpr (kSame) {
      own_dg = own_sum[t].x;
      own_db = own_sum[t].y;
    }
  }
  if (kSame && rows.own >= 0) {
    out[rows.own] = own_dg;
    if constexpr (kLayer) out[a.hidden + rows.own] = own_db;
  }
#pragma unroll
  for (int e = 0; e < N / 2; ++e) {
    const float2 v = halves(kShared || kGroups > 1 ? mine[e * TPR + t] : dg[e]);
    float2 b = make_float2(0.0f, 0.0f);
    if constexpr (kLayer) b = halves(kShared || kGroups > 1 ? mine[(N / 2 + e) * TPR + t] : db[e]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      int c = Part::column(2 * e + j, t, TPR);
      if (c >= rows.body) continue;
      c += rows.head;
      out[c] = j ? v.y : v.x;
      if constexpr (kLayer) out[a.hidden + c] = j ? b.y : b.x;
    }
  }
}

// The CTAs' sums of each column, in the order of the CTAs: kParts parts of them, each in
// order, then the parts.  Latency: few loads a thread where there are few columns, else as few
// CTAs as run at once (4099 x 5001 with both sums 51.6 us with 32 parts, 49.2 with 16).
// (`partial` is still written when this kernel starts: no __restrict__)
constexpr int kWideSums = 2048;
template <int kParts>
__global__ void __launch_bounds__(32 * kParts)
    norm_grad_sum_kernel(const float *partial, int ctas, int columns, int hidden, float *dweight,
                         float *dbias) {
  constexpr int kLoads = 10;
  __shared__ float part[kParts][33];
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  pdl_wait_primary();
  float s = 0.0f;
  if (c < columns) {
    const int per = (ctas + kParts - 1) / kParts, end = min(ctas, (k + 1) * per);
    const float *from = partial + c;
    for (int i0 = k * per; i0 < end; i0 += kLoads) {
      float v[kLoads];
#pragma unroll
      for (int j = 0; j < kLoads; ++j) v[j] = i0 + j < end ? __ldcg(from + (int64_t)(i0 + j) * columns) : 0.0f;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) s += v[j];
    }
  }
  part[k][lane] = s;
  __syncthreads();
  if (k == 0 && c < columns) {
#pragma unroll
    for (int i = 1; i < kParts; ++i) s += part[i][lane];
    if (c < hidden) dweight[c] = s;
    else if (dbias) dbias[c - hidden] = s;
  }
}

int grad_ctas(int rows, int tpr) {
  const int block = tpr == 32 ? kBlock<32> : kBlock<64>, groups = block / tpr, most = kSms * (512 / block);
  // (at least a row for every group, and a CTA for every class of rows)
  const int least = rows < kClasses ? rows : kClasses, ctas = (rows + groups - 1) / groups;
  return ctas < least ? least : ctas < most ? ctas : most;
}

template <typename T, int V, Form kForm, int TPR, int N, bool kLayer>
cudaError_t norm_rows(const T *x, const NormArgs &a, T *y, cudaStream_t stream) {
  // at least a row for every group
  constexpr int kGroups = kNormBlock<TPR> / TPR;
  const int most = kSms * (512 / kNormBlock<TPR>), least = a.rows < kClasses ? a.rows : kClasses;
  int ctas = (a.rows + kGroups - 1) / kGroups;
  ctas = kForm != kAligned && ctas < least ? least : ctas < most ? ctas : most;
  constexpr int kStored = N > 16 ? 2 * N * TPR * 4 : 0;
  auto kernel = norm_kernel<T, V, kForm, TPR, N, kLayer>;
  if (kStored) {
    static std::atomic<uint64_t> ready{0};
    const cudaError_t err = allow_shared(ready, (const void *)kernel, kStored);
    if (err != cudaSuccess) return err;
  }
  kernel<<<ctas, kNormBlock<TPR>, kStored, stream>>>(x, a, y);
  return cudaGetLastError();
}

template <typename T, int V, Form kForm, int TPR, int N, bool kLayer>
cudaError_t grad_rows(const T *dy, const T *x, const GradArgs &a, T *dx, float *dweight,
                      float *dbias, cudaStream_t stream) {
  const int ctas = grad_ctas(a.rows, TPR);
  constexpr bool kHeld = kSumsShared<T, kForm, N, kLayer> || kBlock<TPR> > TPR;
  constexpr size_t smem = (size_t)((kHeld ? kLayer ? 2 : 1 : 0) + (kWeightsShared<kForm, N, kLayer> ? 1 : 0)) * N * TPR * 4;
  auto kernel = norm_grad_kernel<T, V, kForm, TPR, N, kLayer>;
  if (N >= 16 && smem) {  // (with the static arrays it may be above 48 KB)
    static std::atomic<uint64_t> ready{0};
    const cudaError_t err = allow_shared(ready, (const void *)kernel, (int)smem);
    if (err != cudaSuccess) return err;
  }
  kernel<<<ctas, kBlock<TPR>, smem, stream>>>(dy, x, a, dx);
  const cudaError_t err = cudaGetLastError();
  if (err != cudaSuccess) return err;
  const int columns = (kLayer ? 2 : 1) * a.hidden;
  const dim3 grid((columns + 31) / 32);
  return columns < kWideSums ? launch_chained(norm_grad_sum_kernel<32>, grid, dim3(1024), 0, stream, 1, true, a.partial, ctas,
                                              columns, a.hidden, dweight, dbias)
                             : launch_chained(norm_grad_sum_kernel<16>, grid, dim3(512), 0, stream, 1, true, a.partial, ctas,
                                              columns, a.hidden, dweight, dbias);
}

// Calls f.template run<T, V, form>() for a row's type and alignment: 16 bytes an access,
// by windows where rows are not aligned (bf16), or an element an access (fp32, which
// a warp's accesses take whole lines of all the same).
template <typename F>
cudaError_t dispatch(int dtype, bool aligned, bool alike, const F &f) {
  if (dtype == SLIMWISE_DTYPE_BF16)
    return aligned ? f.template run<__nv_bfloat16, 8, kAligned>()
           : alike ? f.template run<__nv_bfloat16, 8, kAlike>()
                   : f.template run<__nv_bfloat16, 8, kAnywhere>();
  return aligned ? f.template run<float, 4, kAligned>() : f.template run<float, 1, kAligned>();
}

// Whether each row starts at one distance from a 16-byte boundary in all n tensors.
bool rows_alike(int element_bytes, int n, const void *const *base, const int64_t *stride) {
  const int v = 16 / element_bytes;
  bool ok = true;
  for (int i = 1; i < n; ++i)
    ok = ok && (reinterpret_cast<uintptr_t>(base[i]) - reinterpret_cast<uintptr_t>(base[0])) % 16 == 0 &&
         (stride[i] - stride[0]) % v == 0;
  return ok;
}

template <bool kLayer>
struct NormCall {
  const void *x;
  NormArgs a;
  void *y;
  cudaStream_t stream;
  template <typename T, int V, Form kForm, int TPR, int N>
  cudaError_t rows() const {
    return norm_rows<T, V, kForm, TPR, N, kLayer>(static_cast<const T *>(x), a, static_cast<T *>(y), stream);
  }
  template <typename T, int V, Form kForm>
  cudaError_t run() const {
    return a.hidden <= 256    ? rows<T, V, kForm, 32, 8>()
           : a.hidden <= 512  ? rows<T, V, kForm, 32, 16>()
           : a.hidden <= 1024 ? rows<T, V, kForm, 64, 16>()
           : a.hidden <= 2048 ? rows<T, V, kForm, 128, 16>()
           : a.hidden <= 4096 ? rows<T, V, kForm, 256, 16>()
           : a.hidden <= 8192  ? rows<T, V, kForm, 512, 16>()
           : a.hidden <= 12288 ? rows<T, V, kForm, 512, 24>()
                               : rows<T, V, kForm, 512, 32>();
  }
};

template <bool kLayer>
struct GradCall {
  const void *dy, *x;
  GradArgs a;
  void *dx;
  float *dweight, *dbias;
  cudaStream_t stream;
  template <typename T, int V, Form kForm, int TPR, int N>
  cudaError_t rows() const {
    return grad_rows<T, V, kForm, TPR, N, kLayer>(static_cast<const T *>(dy), static_cast<const T *>(x), a,
                                           static_cast<T *>(dx), dweight, dbias, stream);
  }
  template <typename T, int V, Form kForm>
  cudaError_t run() const {
    return a.hidden <= 256    ? rows<T, V, kForm, 32, 8>()
           : V == 8 && a.hidden <= 512 ? rows<T, V, kForm, 32, V == 8 ? 16 : 8>()
           : a.hidden <= 1024 ? rows<T, V, kForm, 128, 8>()
           : a.hidden <= 2048 ? rows<T, V, kForm, 256, 8>()
           : a.hidden <= 4096 ? rows<T, V, kForm, V == 8 ? 256 : 512, V == 8 ? 16 : 8>()
           : V < 8 && a.hidden <= 6144 ? rows<T, V, kForm, 512, V < 8 ? 12 : 16>()
           : a.hidden <= 8192  ? rows<T, V, kForm, 512, 16>()
           : a.hidden <= 12288 ? rows<T, V, kForm, 512, 24>()
                               : rows<T, V, kForm, 512, 32>();
  }
};

}  // namespace

cudaError_t launch_norm(const void *x, int dtype, int rows, int hidden, int64_t stride,
                        const float *weight, const float *bias, bool layer, float eps, void *y,
                        int64_t y_stride, float *mean, float *rstd, cudaStream_t stream) {
  const void *base[2] = {x, y};
  const int64_t strides[2] = {stride, y_stride};
  const bool v = rows_aligned(dtype == SLIMWISE_DTYPE_BF16 ? 2 : 4, hidden, 2, base, strides);
  const bool alike = rows_alike(dtype == SLIMWISE_DTYPE_BF16 ? 2 : 4, 2, base, strides);
  const auto extent = [&](const void *p, int64_t step) {
    return dtype == SLIMWISE_DTYPE_BF16 ? extent_of(static_cast<const __nv_bfloat16 *>(p), rows, step, hidden)
                                        : extent_of(static_cast<const float *>(p), rows, step, hidden);
  };
  const NormArgs a = {rows, hidden, extent(x, stride), stride, y_stride, weight, bias, eps, mean, rstd};
  return layer ? dispatch(dtype, v, alike, NormCall<true>{x, a, y, stream})
               : dispatch(dtype, v, alike, NormCall<false>{x, a, y, stream});
}

size_t norm_grad_workspace(int rows, int hidden) {
  // (of either type; groups of 512 threads have the most CTAs but for those of a warp)
  const int narrow = hidden <= 512 ? grad_ctas(rows, 32) : 0, wide = grad_ctas(rows, 512);
  return (size_t)(narrow > wide ? narrow : wide) * 2 * hidden * sizeof(float);
}

cudaError_t launch_norm_grad(const void *dy, int64_t dy_stride, const void *x, int dtype, int rows,
                             int hidden, int64_t stride, const float *weight, const float *mean,
                             const float *rstd, void *dx, int64_t dx_stride, float *dweight,
                             float *dbias, void *workspace, cudaStream_t stream) {
  const void *base[3] = {dy, x, dx};
  const int64_t strides[3] = {dy_stride, stride, dx_stride};
  const bool v = rows_aligned(dtype == SLIMWISE_DTYPE_BF16 ? 2 : 4, hidden, 3, base, strides);
  const bool alike = rows_alike(dtype == SLIMWISE_DTYPE_BF16 ? 2 : 4, 3, base, strides);
  const auto extent = [&](const void *p, int64_t step) {
    return dtype == SLIMWISE_DTYPE_BF16 ? extent_of(static_cast<const __nv_bfloat16 *>(p), rows, step, hidden)
                                        : extent_of(static_cast<const float *>(p), rows, step, hidden);
  };
  const GradArgs a = {rows, hidden, extent(dy, dy_stride), extent(x, stride), dy_stride, stride, dx_stride, weight, mean, rstd,
                      static_cast<float *>(workspace)};
  return mean ? dispatch(dtype, v, alike, GradCall<true>{dy, x, a, dx, dweight, dbias, stream})
              : dispatch(dtype, v, alike, GradCall<false>{dy, x, a, dx, dweight, dbias, stream});
}

}  // namespace slimwise
