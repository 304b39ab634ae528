// sample.cu -- one token per row of logits, drawn with a given random number
// under the row's temperature, top-k, top-p and min-p.
//
// With z' = z / T and m the largest logit, an element's weight is the whole
// number w = floor(2^40 exp((z - m) / T)).  Masses are then sums of whole
// numbers, so that no result depends on how a row was split or in which order
// it was summed, and a draw is the same on every batch size.  In order of
// value (ties: lower id):
//   top-k  the first k elements, of mass M
//   top-p  those of them before which less than p M lies (the first always)
//   min-p  those of them with exp((z - m) / T) >= min_p
// and the token is the first id, ascending, at which the kept mass exceeds
// u times its total.  p and u are taken in 24 bits.
//
// Nearly every row is decided by its best few elements, which the scan of
// vocab.cuh finds in the one read that bounds this kernel.  The mass of the
// whole row, which a nucleus without top-k needs, comes from the same read as a
// float.  Rows that keep more than the listed elements (a wide nucleus, no filter
// at all), and those few whose nucleus would end within that float's error bound,
// are left to the end and then searched by a whole cluster, or by a CTA each where
// they are many: the limits of top-k and top-p by a radix selection of 11 bits a
// pass over the row, from histograms of masses and counts, then the token by a
// running sum over ids.  Where clusters scan the rows, the same kernel does that;
// where single CTAs do, a second kernel, so that a left-over row still gets a
// cluster and the first keeps four CTAs on an SM.
//
// 512 rows of 262144 bf16 under mixed requests: 68 us, 3.9 TB/s, four rows on some
// SMs and three on others (47 us at the least); 256 of 150001 fp32 43 us, 3.6 TB/s,
// one or two rows on an SM.  What takes the rest of both is not established: issue
// slots are 36 and 64 % busy, DRAM 52 and 53 %, and more copies in flight (a third
// stage of the rings) gain nothing.  64 rows of 131072 fp32 with top-p 22.5 us, one
// row 15 us: one after the other a launch, the scan, the join and the decision.  A
// search costs more: 512 rows of 131072 bf16 without any filter 128 us (by its
// instructions), with top-k 1000 475, with a nucleus of 0.9 of nearly flat rows 0.9
// ms (the histograms' atomics in shared memory); its functions spill up to 164 bytes
// a thread.
#include "vocab.cuh"

namespace slimwise {

// Three stages of the rings, as top logits have for few rows, gain nothing here
// (200 rows of 150001 bf16 29.8 us against 28.0).  256 rows of 150001 fp32 take 38
// us with three CTAs on an SM, which leave the scan its registers, and 46 with
// four; 512 of 262144 bf16, which four hold at once, 73 and 67.
constexpr int kSampleStages = kManyStages;
// The search goes by the same rule.  With all rows left over, 512 of 131072 bf16
// take 128 us without a filter and 900 with a nucleus of 0.9 of nearly flat rows
// with four CTAs on an SM, 195 and 1390 with three, 163 and 1560 with five; 380 of
// 131072 fp32, which three hold at once, 142 and 836 with three, 162 and 976 with
// four, 150 and 1260 with five.
constexpr int kNucleus = 32;      // elements looked at for a nucleus or min-p without top-k
constexpr int kSampleRoom = 128;  // of a warp's list
constexpr int kTopKListed = kSampleRoom - 32;  // largest top-k that is decided from the list
constexpr int32_t kLeftOver = -2; // a token that is still to be searched (its logprob: the maximum)
constexpr float kWeightOne = 1099511627776.0f;  // 2^40, the largest element's weight
// Bound of the relative difference between the scan's float sum of the elements
// that are not listed and the sum of their weights (but for the weights'
// truncation, one part in 2^40 each).  An element at 2^-x of the largest weighs
// less than its truncation beyond x = 40.  In units of 2^-24, along the longest way
// that an element's share can take:
//   145  exponents of 40 bits: of the scan rounded three times, and the logarithm's
//        base; of the weights twice (the quotient 1 / T is the same in both)
//     8  exp2's and exp's own
//   290  58 changes of a sum's reference, a factor of exp2 and a product: 4 at
//        refreshes, 48 at cuts of a warp's list (3072 units of it, 64 between two
//        cuts), 6 in most_of_many() and the join
//   217  additions of units that are dropped from the list: their factor, and four to
//        a lane at each refresh and cut and at the row's end
//    32  additions of windows, elements and keys in most_of_many() and the join
//    52  of the row's end: windows and elements of the listed units to a lane
//    32  sums of a unit, over steps (compensated), threads and CTAs
//     5  the reference's factor
// which are 781 or less than 2^-14 in all.
constexpr uint64_t kMassError = 1 << 14;  // one part in

// What a search uses of shared memory, where the scan's was.
constexpr int kBins = 2048;
// Rows left over in a cluster's share from which each is searched by one CTA: 608
// rows of 32000 fp32 without a filter (8 a cluster) take 73 us so and 156 by
// clusters, 512 of 131072 bf16 (6 or 7) 128 and 182; with a nucleus of 0.9, 304
// of 131072 bf16 (4) 723 and 610.
constexpr int kAloneFrom = 6;
// Steps of 4 x 32 windows of a warp.
constexpr int kStepsMax = (kVocabMax / 4 / kScanWarps + 127) / 128 + 1;
struct SearchShared {
  uint32_t hist[2][kBins];           // of a pass: two copies of counts, or sums of weights in two halves
  uint64_t slot[2][kClusterMax];     // each CTA's sum
  uint64_t red[kScanWarps];
  uint64_t above;                    // result of a pass, written by the CTA that found it
  int bin;
  uint32_t left[kScanWarps];         // rows that are left over, a bit each
};
static_assert(sizeof(SearchShared) <= sizeof(ScanShared<kSampleStages>), "the search fits the scan's memory");
static_assert(kScanWarps * kStepsMax * 8 <= sizeof(SearchShared::hist), "the steps' sums fit the bins");
struct SampleShared {
  uint64_t weight[kTopMax];
};
struct SampleArgs {
  const float *temperature;
  const int32_t *top_k;
  const float *top_p, *min_p, *uniform;
  int32_t *tokens;
  float *logprob;
};

__device__ __forceinline__ uint64_t fraction(uint64_t mass, uint64_t f24) {
  return ((mass >> 32) * f24 << 8) + ((mass & 0xFFFFFFFFull) * f24 >> 24);
}

struct Draw {  // one row's request
  float inv;   // 1 / T
  float min_p;
  int top_k;   // 1 .. vocab
  uint64_t p24, u24;
  bool limited, nucleus;  // whether top-k, top-p leave anything out
};
__device__ __forceinline__ float element_exp(float z, float m, float inv) {
  return expf(__fmul_rn(__fsub_rn(z, m), inv));
}
// floor(2^40 e) of an e in [0, 1], by shifting its mantissa (a conversion to 64
// bits takes many times as long); what lies under 2^-40 shifts out.
__device__ __forceinline__ uint64_t element_weight(float e) {
  const uint32_t b = __float_as_uint(e), mantissa = (b & 0x7FFFFFu) | 0x800000u;
  const int shift = (int)(b >> 23) - (127 + 23 - 40);
  return shift >= 0 ? (uint64_t)mantissa << shift : (uint64_t)(mantissa >> min(-shift, 31));
}

// The CTAs that search a row: all of a cluster, or one of it.
struct Team {
  int C, rank;  // CTAs, this one's place
  __device__ __forceinline__ void sync() const {
    if (C > 1) cg::this_cluster().sync();
    else __syncthreads();
  }
  template <typename V>
  __device__ __forceinline__ V *of(V *p, int r) const {
    return C > 1 ? cg::this_cluster().map_shared_rank(p, r) : p;
  }
};

// Sum of a whole number over the team; slot[parity] keeps each CTA's.
__device__ __forceinline__ uint64_t team_sum(const Team team, uint64_t v, int &parity, SearchShared &sh) {
  const int tid = threadIdx.x;
  v = block_reduce<kScanThreads>(v, sh.red, OpAdd());
  if (tid < team.C) *team.of(&sh.slot[parity][team.rank], tid) = v;
  team.sync();
  v = 0;
  for (int r = 0; r < team.C; ++r) v += sh.slot[parity][r];
  parity ^= 1;
  return v;
}

// The part of a row that this CTA passes over.
template <typename T>
struct Part {
  Row<T> row;
  Team team;
  int lo, hi;
  float m, inv;
  // f(window, its number) of windows i, i + step, ... of U (none beyond end: of
  // -inf), all loaded before the first f; f's code is there once.
  static constexpr int U = 4;
  template <typename F>
  __device__ __forceinline__ void batch(int i, int step, int end, F f) const {
    uint4 v[U];
    const uint32_t none = neg_inf_bits(row.p);
    if (i >= row.whole_lo && i + (U - 1) * step < min(end, row.whole_lo + row.whole_n)) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = ld_global_v4(row.w + i + u * step);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = make_uint4(none, none, none, none);
#pragma unroll 1
      for (int u = 0; u < U; ++u) {
        const uint4 w = i + u * step < end ? load_window(row, i + u * step) : make_uint4(none, none, none, none);
#pragma unroll
        for (int x = 0; x < U; ++x)
          if (x == u) v[x] = w;
      }
    }
#pragma unroll 1
    for (int u = 0; u < U; ++u) {
      f(v[0], i + u * step);
#pragma unroll
      for (int x = 0; x + 1 < U; ++x) v[x] = v[x + 1];
    }
  }
  // f(element, id) of all elements of this CTA's part.  (Elements beside the row
  // are -inf: they weigh nothing, and come with ids outside the row.)
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    constexpr int E = Row<T>::E;
    for (int i = lo + (int)threadIdx.x; i < hi; i += U * kScanThreads)
      batch(i, kScanThreads, hi, [&](const uint4 &v, int at) {
        float z[E];
        unpack<T>(v, z);
        const int id0 = at * E - row.mis;
#pragma unroll
        for (int e = 0; e < E; ++e) f(z[e], id0 + e);
      });
  }
};

// A prefix of the order: values above `o`, and of those equal to it the ids up
// to `id`.
struct Limit {
  uint32_t o;
  int id;
  __device__ __forceinline__ bool has(uint32_t v, int i) const { return v > o || (v == o && i <= id); }
};

// What the elements of a row count for in a running sum: (z, id), and a whole
// window's from id0 on.
struct EqualTo {  // one if they are o, as ordered(), and in the row
  uint32_t o;
  int vocab;
  __device__ __forceinline__ uint64_t operator()(float z, int id) const {
    return ordered(z) == o && (unsigned)id < (unsigned)vocab;
  }
  template <int E>
  __device__ __forceinline__ uint64_t window(const float (&z)[E], int id0) const {
    uint32_t n = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) n += (*this)(z[e], id0 + e) ? 1 : 0;
    return n;
  }
};
template <bool kAll>
struct KeptWeight {  // their weights, if they are kept (kAll: all are)
  Limit keep;
  float m, inv, min_p;
  __device__ __forceinline__ float kept(float z, int id) const {
    const float e = element_exp(z, m, inv);
    return kAll || (keep.has(ordered(z), id) && e >= min_p) ? e : 0.0f;
  }
  __device__ __forceinline__ uint64_t operator()(float z, int id) const { return element_weight(kept(z, id)); }
  // floor(2^40 e) as two whole numbers of 20 bits, which a sum with 2^23, rounded
  // down, leaves in a float's low bits: floor(2^20 e), and that of the remainder,
  // which is exact.  Half as many instructions as the shift to 64 bits takes.
  template <int E>
  __device__ __forceinline__ uint64_t window(const float (&z)[E], int id0) const {
    constexpr float kUnit = 1048576.0f, kOnes = 8388608.0f;
    uint32_t high = 0, low = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float k = kept(z[e], id0 + e), h = __fmaf_rd(k, kUnit, kOnes);
      const float l = __fmaf_rd(__fmaf_rn(k, kUnit, kOnes - h), kUnit, kOnes);
      high += __float_as_uint(h);
      low += __float_as_uint(l);
    }
    constexpr uint32_t kBias = 0x4B000000u * E;  // (modulo 2^32)
    return ((uint64_t)(high - kBias) << 20) + (low - kBias);
  }
};

// Bins of a pass: counts, or masses (kMass), of the elements within `in` whose bits
// from `known` up are the prefix's, by their bits from `shift` to there.  A
// function of its own (inlined, top-k 1000 of 512 x 131072 bf16 took 531 us, not 475).
template <bool kMass, typename T>
__device__ __noinline__ void histogram(const Part<T> part, const Limit in, int known, int shift,
                                       uint32_t prefix, SearchShared &sh) {
  const int tid = threadIdx.x, copy = tid & 1;
  for (int i = tid; i < 2 * kBins; i += kScanThreads) (&sh.hist[0][0])[i] = 0;
  __syncthreads();
  const uint32_t mask = (1u << (known - shift)) - 1u, others = known < 32 ? ~0u << known : 0;
  part.each([&](float z, int id) {
    const uint32_t o = ordered(z);
    if (!in.has(o, id) || ((o ^ prefix) & others) || (unsigned)id >= (unsigned)part.row.vocab) return;
    const uint32_t bin = o >> shift & mask;
    if constexpr (kMass) {
      const uint64_t w = element_weight(element_exp(z, part.m, part.inv));
      // a sum of 64 bits in two, by hand: few weights have a high half
      const uint32_t low = (uint32_t)w, was = low ? atomicAdd(&sh.hist[0][bin], low) : 0;
      const uint32_t high = (uint32_t)(w >> 32) + (was + low < was);
      if (high) atomicAdd(&sh.hist[1][bin], high);
    } else {
      atomicAdd(&sh.hist[copy][bin], 1u);  // (two copies: fewer lanes meet)
    }
  });
}

// The largest value v (as ordered()) with amount(values >= v within `in`) at
// least `want`, and in `above` the amount of the values > v.  Amounts are weights
// (kMass) or counts.  want 0: the share p24 of the whole amount; cut: that wanted.
template <bool kMass, typename T>
__device__ __noinline__ uint32_t search_value(const Part<T> part, Limit in, uint64_t want,
                                              uint64_t p24, uint64_t &above, uint64_t &cut, int &parity,
                                              SearchShared &sh) {
  const Team team = part.team;
  const int C = team.C, rank = team.rank;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = kBins / C, mine = per / kScanThreads;  // bins of a CTA, of a thread
  uint32_t prefix = 0;
  above = 0;
  for (int known = 32; known > (sizeof(T) == 2 ? 16 : 0);) {
    const int shift = max(known - 11, sizeof(T) == 2 ? 16 : 0);  // (a bf16 has 16 bits)
    histogram<kMass>(part, in, known, shift, prefix, sh);
    team.sync();
    // CTA r joins bins r per .. of all CTAs, each thread `mine` of them
    const int first = rank * per + tid * mine;
    uint64_t amount[kBins / kScanThreads], sum = 0;
#pragma unroll
    for (int j = 0; j < kBins / kScanThreads; ++j) {
      amount[j] = 0;
      if (j < mine)
        for (int r = 0; r < C; ++r) {
          const uint32_t *const h = team.of(&sh.hist[0][first + j], r);
          amount[j] += h[0] + ((uint64_t)h[kBins] << (kMass ? 32 : 0));
        }
      sum += amount[j];
    }
    // this thread's higher bins' amount within the CTA, then the cluster
    uint64_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t v = __shfl_down_sync(0xFFFFFFFFu, incl, o);
      if (lane + o < 32) incl += v;
    }
    if (lane == 0) sh.red[warp] = incl;
    __syncthreads();
    uint64_t over = incl - sum, total = 0;
    for (int w = 0; w < kScanWarps; ++w) {
      if (w > warp) over += sh.red[w];
      total += sh.red[w];
    }
    if (tid < C) *team.of(&sh.slot[parity][rank], tid) = total;
    team.sync();
    uint64_t all = 0;
    for (int r = 0; r < C; ++r) {
      if (r > rank) over += sh.slot[parity][r];
      all += sh.slot[parity][r];
    }
    parity ^= 1;
    if (want == 0) {
      want = fraction(all, p24);
      if (want < 1) want = 1;
    }
    if (known == 32) cut = want;
#pragma unroll
    for (int j = kBins / kScanThreads - 1; j >= 0; --j) {
      if (j >= mine) continue;
      if (over < want && want <= over + amount[j])
        for (int r = 0; r < C; ++r) {
          *team.of(&sh.above, r) = over;
          *team.of(&sh.bin, r) = first + j;
        }
      over += amount[j];
    }
    team.sync();
    prefix |= (uint32_t)sh.bin << shift;
    above += sh.above;
    want -= sh.above;
    known = shift;
  }
  // the other bits of a bf16: its own are inverted below zero
  return sizeof(T) == 2 && !(prefix >> 31) ? prefix | 0xFFFFu : prefix;
}

// The first id at which the running sum over ids of f(element, id) exceeds
// target(the sum over all), by the thread that has it: found(id, f there, sum).
// CTAs' warps take consecutive runs of windows, so that the running sum is one
// over CTAs, warps, steps of 4 x 32 windows, those 4, lanes and elements.
template <typename T, typename F, typename G, typename H>
__device__ __forceinline__ void search_sum(const Part<T> &part, const F f, G target_of, H found,
                                           int &parity, SearchShared &sh) {
  constexpr int E = Row<T>::E;
  const int rank = part.team.rank;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (part.hi - part.lo + kScanWarps - 1) / kScanWarps;
  const int lo = min(part.lo + warp * per, part.hi), hi = min(lo + per, part.hi);
  // each step's sum is kept, so that only the step of the target is read again
  uint64_t *const steps = reinterpret_cast<uint64_t *>(sh.hist) + warp * kStepsMax;
  auto window_sum = [&](const uint4 &v, int i) {
    float z[E];
    unpack<T>(v, z);
    return f.window(z, i * E - part.row.mis);
  };
  uint64_t mine = 0;
  constexpr int U = Part<T>::U;
  for (int i = lo, k = 0; i < hi; i += 32 * U, ++k) {
    uint64_t s = 0;
    part.batch(i + lane, 32, hi, [&](const uint4 &v, int at) { s += window_sum(v, at); });
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (lane == 0) steps[k] = s;
    mine += s;
  }
  const int at = parity;
  const uint64_t total = team_sum(part.team, lane == 0 ? mine : 0, parity, sh);
  const uint64_t target = target_of(total);
  if (lane == 0) sh.red[warp] = mine;
  __syncthreads();
  uint64_t before = 0;
  for (int r = 0; r < rank; ++r) before += sh.slot[at][r];
  for (int w = 0; w < warp; ++w) before += sh.red[w];
  if (target < before || target >= before + mine) return;
  int i = lo;
  for (int k = 0; before + steps[k] <= target; ++k, i += 32 * U) before += steps[k];
  part.batch(i + lane, 32, hi, [&](const uint4 &v, int at) {
    const uint64_t s = window_sum(v, at);
    uint64_t incl = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t more = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += more;
    }
    uint64_t b = before + incl - s;
    before += __shfl_sync(0xFFFFFFFFu, incl, 31);
    if (target >= b && target < b + s) {
      float z[E];
      unpack<T>(v, z);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint64_t w = f(z[e], at * E - part.row.mis + e);
        if (target >= b && target < b + w) found(at * E - part.row.mis + e, w, total);
        b += w;
      }
    }
  });
}

// The id up to which there are `want` elements of value o.
template <typename T>
__device__ __noinline__ int search_id(const Part<T> part, uint32_t o, uint64_t want, int &parity,
                                      SearchShared &sh) {
  const Team team = part.team;
  search_sum(
      part, EqualTo{o, part.row.vocab},
      [&](uint64_t) { return want - 1; },
      [&](int id, uint64_t, uint64_t) {
        for (int r = 0; r < team.C; ++r) *team.of(&sh.bin, r) = id;
      },
      parity, sh);
  team.sync();
  return sh.bin;
}

// The token among the elements that are kept.
template <typename T, typename F>
__device__ __noinline__ void search_token(const Part<T> part, const F f, uint64_t u24, int &parity,
                                          int32_t *token, float *logprob, SearchShared &sh) {
  search_sum(
      part, f, [&](uint64_t total) { return fraction(total, u24); },
      [&](int id, uint64_t w, uint64_t total) {
        *token = id;
        *logprob = logf((float)w / (float)total);
      },
      parity, sh);
}

// The whole request over the whole row, by all CTAs of the team.
template <typename T>
__device__ __noinline__ void search_row(const Part<T> part, const Draw d, int &parity,
                                        int32_t *token, float *logprob, SearchShared &sh) {
  Limit keep = {0, part.row.vocab};
  uint64_t above, cut;
  if (d.limited) {
    keep.o = search_value<false>(part, keep, (uint64_t)d.top_k, 0, above, cut, parity, sh);
    keep.id = search_id(part, keep.o, (uint64_t)d.top_k - above, parity, sh);
  }
  if (d.nucleus) {
    // of the elements of value o (each of weight w > 0), those before which less
    // than the cut lies; top-k's limit already holds among them
    const uint32_t o = search_value<true>(part, keep, 0, d.p24, above, cut, parity, sh);
    const uint64_t w = element_weight(element_exp(unordered(o), part.m, part.inv));
    const int id = search_id(part, o, (cut - above + w - 1) / w, parity, sh);
    keep.id = o == keep.o ? min(id, keep.id) : id;
    keep.o = o;
  }
  if (d.limited || d.nucleus || d.min_p > 0.0f)
    search_token(part, KeptWeight<false>{keep, part.m, part.inv, d.min_p}, d.u24, parity, token, logprob, sh);
  else
    search_token(part, KeptWeight<true>{keep, part.m, part.inv, d.min_p}, d.u24, parity, token, logprob, sh);
}

// The request decided at a row's leader from its n largest elements, sh.cand;
// false if they do not decide it.  rest: the sum of 2^((z - ref) c) over all
// other elements; m: the row's maximum.
template <typename S>
__device__ __forceinline__ bool decide(const Draw &d, int n, float rest, float ref, float c, float m,
                                       int vocab, int32_t *token, float *logprob, S &sh, SampleShared &sm) {
  const int tid = threadIdx.x;
  // a few lanes for each candidate; the first of them holds it
  const int lanes = candidate_lanes(n), at = tid / lanes, sub = tid % lanes;
  if (tid < n) sm.weight[tid] = element_weight(element_exp(key_value(sh.cand[tid]), m, d.inv));
  uint64_t key = at < n ? sh.cand[at] : 0;
  __syncthreads();
  int rank = 0;
  uint64_t before = 0;
  if (key) {
#pragma unroll 4
    for (int i = sub; i < n; i += lanes) {
      const bool first = sh.cand[i] > key;
      rank += first;
      before += first ? sm.weight[i] : 0;
    }
  }
  for (int o = 1; o < lanes; o *= 2) {
    rank += __shfl_xor_sync(0xFFFFFFFFu, rank, o);
    before += __shfl_xor_sync(0xFFFFFFFFu, before, o);
  }
  const uint64_t shared_key = key;
  if (sub) key = 0;
  const float e = key ? element_exp(key_value(key), m, d.inv) : 0.0f;
  uint64_t w = key ? sm.weight[at] : 0;
  const bool in = key && rank < d.top_k;
  const uint64_t listed = block_reduce<kScanThreads>(in ? w : 0, sh.red64, OpAdd());
  uint64_t cut = ~0ull;
  if (n >= d.top_k) {
    if (d.nucleus) cut = fraction(listed, d.p24);
  } else {
    // the elements that are not listed come after these; with both limits, the
    // nucleus is one of a mass that is not known here
    if (d.limited && d.nucleus) return false;
    const float last = -block_reduce<kScanThreads>(key ? -e : -INFINITY, sh.redf, OpMax());
    uint64_t low = ~0ull;
    if (d.nucleus) {
      // the mass: the listed elements', which are all the largest, and about the rest's
      const uint64_t about = __float2ull_rz(rest * ex2((ref - m) * c) * kWeightOne);
      const uint64_t error = about / kMassError + (uint64_t)vocab + 2;
      low = fraction(listed + about - min(about, error), d.p24);
      cut = fraction(listed + about + error, d.p24) + 1;
    }
    if (!(last < d.min_p) && (!d.nucleus || listed < cut)) return false;
    if (__syncthreads_or(key && rank > 0 && before >= low && before < cut)) return false;
  }
  if (cut < 1) cut = 1;
  if (!(in && before < cut && e >= d.min_p)) w = 0;
  __syncthreads();
  if (key) sm.weight[at] = w;
  const uint64_t total = block_reduce<kScanThreads>(w, sh.red64, OpAdd());
  const uint64_t target = fraction(total, d.u24);
  uint64_t id_before = 0;
  if (shared_key) {
#pragma unroll 4
    for (int i = sub; i < n; i += lanes)  // (the key's low half is the complement of the id)
      id_before += (uint32_t)sh.cand[i] > (uint32_t)shared_key ? sm.weight[i] : 0;
  }
  for (int o = 1; o < lanes; o *= 2) id_before += __shfl_xor_sync(0xFFFFFFFFu, id_before, o);
  if (w && target >= id_before && target < id_before + w) {
    *token = (int32_t)key_index(key);
    *logprob = logf((float)w / (float)total);
  }
  return true;
}

// The request of row t, and how many elements to look at: all that top-k leaves,
// else a guess of what a nucleus or min-p keeps; without any filter only the
// largest.  False if the request is out of range.
__device__ __forceinline__ bool request_of(const SampleArgs &a, int t, int vocab, Draw &d, int &K) {
  const float temp = a.temperature ? a.temperature[t] : 1.0f;
  const int tk = a.top_k ? a.top_k[t] : 0;
  const float tp = a.top_p ? a.top_p[t] : 1.0f;
  const float mp = a.min_p ? a.min_p[t] : 0.0f;
  const float u = a.uniform[t];
  const bool good = temp >= 0.0f && temp < INFINITY && tp >= 0.0f && mp <= 1.0f && u >= 0.0f && u < 1.0f;
  const bool greedy = !good || temp < FLT_MIN;
  d.inv = greedy ? 1.0f : 1.0f / temp;
  d.min_p = mp;
  d.top_k = greedy ? 1 : (tk > 0 && tk < vocab) ? tk : vocab;
  d.limited = d.top_k < vocab;
  d.nucleus = tp < 1.0f;
  d.p24 = (uint64_t)(fminf(tp, 1.0f) * 16777216.0f);
  d.u24 = (uint64_t)(u * 16777216.0f);
  K = d.top_k <= kTopKListed ? d.top_k : (d.nucleus || mp > 0.0f) ? min(kNucleus, vocab) : 1;
  return good;
}

// Row t's token, by its leader's threads, from its n largest elements in sh.cand
// and s, this thread's part of the sum of all others.  Not inlined: the scan's
// loop keeps its registers.
template <typename T, typename S>
__device__ __noinline__ void finish_row(const SampleArgs &a, const Row<T> row, int t, int n, float s,
                                        float ref, S &sh, SampleShared &sm) {
  const int tid = threadIdx.x;
  Draw d;
  int K;
  const bool good = request_of(a, t, row.vocab, d, K);
  const float c = kLog2e * d.inv;
  const float m = block_reduce<kScanThreads>(tid < n ? key_value(sh.cand[tid]) : -INFINITY, sh.redf, OpMax());
  const float rest = block_reduce<kScanThreads>(s, sh.redf, OpAdd());
  if (!good || !(rest < INFINITY) || !(m > -INFINITY) || !(m < INFINITY)) {
    // NaN or +inf in the row, or nothing but -inf: no distribution
    if (tid == 0) {
      a.tokens[t] = -1;
      a.logprob[t] = NAN;
    }
    return;
  }
  if (!decide(d, n, rest, ref, c, m, row.vocab, a.tokens + t, a.logprob + t, sh, sm) && tid == 0) {
    a.tokens[t] = kLeftOver;
    a.logprob[t] = m;
  }
}

// The rows of this cluster that were left over: a few are searched by all its
// CTAs, one after the other; if they are many (kAlone), by a CTA each.
template <typename T, bool kAlone>
__device__ __forceinline__ void search_rows(const T *logits, int64_t stride, int rows, int vocab,
                                            const SampleArgs &a, SearchShared &sh) {
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, first = (int)(blockIdx.x / C), clusters = (int)(gridDim.x / C);
  int parity = 0;
  for (int base = first; base < rows; base += kScanThreads * clusters) {
    // (a row's own search writes its token after a barrier that all CTAs reach)
    const int mine = base + tid * clusters;
    const bool left = mine < rows && __ldcg(a.tokens + mine) == kLeftOver;
    const uint32_t mask = __ballot_sync(0xFFFFFFFFu, left);
    if ((tid & 31) == 0) sh.left[tid >> 5] = mask;
    const int n = __syncthreads_count(left);
    if (n == 0) continue;
    const bool alone = kAlone && n >= kAloneFrom;
    const Team team = {alone ? 1 : C, alone ? 0 : rank};
    if (alone) cluster.sync();
    int turn = 0;
    for (int w = 0; w < kScanWarps; ++w)
      for (uint32_t bits = sh.left[w]; bits; bits &= bits - 1) {
        if (alone && turn++ % C != rank) continue;
        const int t = base + (32 * w + __ffs((int)bits) - 1) * clusters;
        Draw d;
        int K;
        request_of(a, t, vocab, d, K);
        Part<T> part = {Row<T>(logits + (int64_t)t * stride, vocab), team, 0, 0, __ldcg(a.logprob + t), d.inv};
        const int per = (part.row.windows + team.C - 1) / team.C;
        part.lo = min(team.rank * per, part.row.windows);
        part.hi = min(part.lo + per, part.row.windows);
        search_row(part, d, parity, a.tokens + t, a.logprob + t, sh);
        __syncthreads();  // the next row's bins lie where this one's steps are read
      }
    if (alone) {
      cluster.sync();  // before others write here again
      parity = 0;      // (each CTA's rows took another number of sums)
    } else {
      __syncthreads();  // every warp has read sh.left to its end
    }
  }
  cluster.sync();  // no CTA ends while its sums can still be read or written
}

template <typename T, bool kCluster, int kCtas>
__global__ void __launch_bounds__(kScanThreads, kCtas)
    sample_kernel(const T *__restrict__ logits, int64_t stride, int rows, int vocab, int K_most,
                  const __grid_constant__ SampleArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  SampleShared &sm = *reinterpret_cast<SampleShared *>(smem);
  auto &sh = *reinterpret_cast<ScanShared<kSampleStages> *>(smem + sizeof(SampleShared));
  if constexpr (!kCluster) pdl_launch_dependents();  // the search kernel, which waits
  Scan<T, kCluster, true, false, kSampleStages> scan(sh, kSampleRoom, K_most, logits, stride, vocab, rows);
  auto request = [&](int t, int &K, float &c, bool &sums) {
    Draw d;
    request_of(a, t, vocab, d, K);
    c = kLog2e * d.inv;
    sums = d.nucleus && !d.limited;  // only such a nucleus is one of the row's whole mass
  };
  scan.rows_of_cluster(request, [&](int t, int n) {
    finish_row(a, scan.row_of(t), t, n, scan.s, scan.ref, sh, sm);
  });
  if constexpr (kCluster) {
    cg::this_cluster().sync();
    search_rows<T, false>(logits, stride, rows, vocab, a, *reinterpret_cast<SearchShared *>(&sh));
  }
}

template <typename T, int kCtas>
__global__ void __launch_bounds__(kScanThreads, kCtas)
    sample_search_kernel(const T *__restrict__ logits, int64_t stride, int rows, int vocab,
                         const __grid_constant__ SampleArgs a) {
  __shared__ SearchShared search;
  pdl_wait_primary();
  search_rows<T, true>(logits, stride, rows, vocab, a, search);
}

template <typename T, bool kCluster, int kCtas>
static cudaError_t launch_scan(const ScanGrid &g, const T *z, int64_t stride, int rows, int vocab, int K_most,
                               const SampleArgs &a, cudaStream_t stream) {
  return launch_clusters<sample_kernel<T, kCluster, kCtas>>(
      g.clusters, g.C, kScanThreads, g.smem,
      sizeof(SampleShared) + scan_smem(kSampleStages, kSampleRoom, kTopKListed, kCluster ? kClusterMax : 1, false),
      stream, z, stride, rows, vocab, K_most, a);
}

template <typename T>
static cudaError_t launch(const void *logits, int rows, int vocab, int64_t stride,
                          const float *temperature, const int32_t *top_k, const float *top_p,
                          const float *min_p, const float *uniform, int32_t *tokens,
                          float *logprob, cudaStream_t stream) {
  const int K_most = top_k ? kTopKListed : kNucleus;
  const ScanGrid g = scan_grid(rows, vocab, (int)sizeof(T), kSampleRoom, K_most, false, kSampleStages,
                               sizeof(SampleShared));
  const SampleArgs a = {temperature, top_k, top_p, min_p, uniform, tokens, logprob};
  const T *const z = static_cast<const T *>(logits);
  const auto launch =
      g.C > 1 ? launch_scan<T, true, kFewCtas>
      : g.few ? launch_scan<T, false, kFewCtas>
              : launch_scan<T, false, kManyCtas>;
  cudaError_t err = launch(g, z, stride, rows, vocab, K_most, a, stream);
  if (err != cudaSuccess || g.C > 1) return err;
  const int clusters = (g.few ? kFewCtas : kManyCtas) * 152 / kClusterMax;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kClusterMax;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((rows < clusters ? rows : clusters) * kClusterMax));
  cfg.blockDim = dim3(kScanThreads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, g.few ? sample_search_kernel<T, kFewCtas> : sample_search_kernel<T, kManyCtas>,
                            z, stride, rows, vocab, a);
}

cudaError_t launch_sample(const void *logits, int dtype, int rows, int vocab, int64_t stride,
                          const float *temperature, const int32_t *top_k, const float *top_p,
                          const float *min_p, const float *uniform, int32_t *tokens,
                          float *logprob, cudaStream_t stream) {
  return dtype == SLIMWISE_DTYPE_BF16
             ? launch<__nv_bfloat16>(logits, rows, vocab, stride, temperature, top_k, top_p, min_p,
                                     uniform, tokens, logprob, stream)
             : launch<float>(logits, rows, vocab, stride, temperature, top_k, top_p, min_p,
                             uniform, tokens, logprob, stream);
}

}  // namespace slimwise
