// mcd_sample_rows (include/mcd_rows.h): one id of every logits row by temperature, top-k, top-p and min-p.
//
// The mathematics is in whole numbers: an id's weight is W = floor(2^31 exp32(logit / T - z_max)), and every filter is a cut of the
// ranking (logit descending, id ascending): "the first k", "until the weights' sum reaches a target", "no weight below".
// A cut is found without sorting: a histogram (counts and sums of W) over 256 equal steps down from the maximum, the bin in which
// the target is crossed, and of that bin's ids each one's sum of those before it (few ids; many are narrowed by histograms of
// their keys first).  The draw is the same on ids in ascending order, its target a sum of weights.
//
// A cluster of CTAs takes a row and reads it for the maximum.  Then one of three ways:
//   top_k up to 128: of as many groups of threads, so many ids are not below the least of the groups' maxima; what is not goes to a
//     list in the first CTA's shared memory, and the first CTA goes on alone;
//   top_k otherwise, top_p: the histogram is made from the row, by all CTAs; the ids of the bins down to the crossing one go to the list,
//     as above; where they are too many, those of the crossing bin alone, while the bins above are summed up, and the draw is from
//     the row.  Where min_p leaves nothing below the crossing bin there is no cut to find;
//   neither: the draw is from the row: sums of W of blocks of 256 ids, the block in which the target is crossed, the id.
// Order never changes a result: whole numbers add up to the same sum.
//
// What bounds it: weights, about 30 operations each (the definition rounds every product and sum), barriers of the cluster (2,000
// cycles each) and chains of small steps.  One row of 2,048, k = 50: 6 us on the GPU; of 131,072: 13 us, with top_p alone and 30,000
// ids left 28 (35 of 8 rows).  128 rows of 2,048 with mixed settings 12.3 us, 96 of 131,072 (bf16) 47 to 51: as long as the rows with
// large sets, a fifth, take beside others.
#pragma once
#include <cooperative_groups.h>

#include <cmath>
#include <type_traits>

#include "mcd_cache.cuh"
#include "mcd_rows.cuh"
#include "mcd_sampler.cuh"

namespace mcd {
namespace rows {

struct SampleArgs {
  const void* logits;
  long long stride;
  int vocab, cluster;
  int n_rows, ordered;                 // rows by what they take
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  const double* u;
  int32_t* ids;
  float* probs;
  int32_t* kept;
  int32_t* err;
};

// The kernel's launch for logits of a type; each type is compiled by a file of its own.
template <class T>
cudaError_t launch_sample(SampleArgs a, int n_rows, cudaStream_t st);

namespace {

namespace cg = cooperative_groups;

constexpr int kMaxWarps = 16;
constexpr int kMostGroups = 128;       // groups of threads, whose maxima bound the largest ids
constexpr int kMaxCluster = 8, kPerSm = 4;
constexpr int kList = 3200;            // ids of the list
constexpr int kFew = 128;              // ids whose order is found by comparing all with all
constexpr int kMaxVocabRows = 1 << 18;
constexpr int kBlocks = kMaxVocabRows / kMaxCluster / 256;      // blocks of 256 ids in a CTA's share

// Keys in the order of the logits (finite ones and -inf): a larger logit has a larger key; -0 is 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// The cluster's barrier, for threads whose warp may not be together at it, and ordered with the memory accesses around it.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}

struct Tally {
  unsigned long long mass;
  uint32_t count;
};
// What a CTA tells the others.
struct Told {
  float top, least;                    // its maximum, the least of its groups' maxima
  int bad, odd;                        // logits that do not fit; that are not quotients' plain operands
  uint32_t lo, hi;
  Tally sum;
};
// A cut of the ranking: what is before it, itself included, is left.
struct Cut {
  uint32_t key, id;
  Tally in;
};

struct Shared {
  uint32_t hist[3][256];               // counts, sums of the low 16 bits of W, of the others
  uint32_t key[kList], id[kList], w[kList];
  uint4 few[kFew];                     // key, id, W
  unsigned long long block[kBlocks];
  uint32_t n_list, n_few;
  Told told[4][kMaxCluster];           // of the maximum, of sums, of extents
  Tally red[kMaxWarps];
  float fred[2][kMaxWarps];
  int flags[kMaxWarps];
  uint32_t ured[2][kMaxWarps];
  uint32_t bin;
  Tally above, at;
  Cut cut;
  uint32_t kinds[3][kMaxWarps], row;
};

__device__ __forceinline__ unsigned long long warp_sum(unsigned long long x) {
#pragma unroll
  for (int w = 16; w; w >>= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
  return x;
}
// The same of numbers below 2^36.
__device__ __forceinline__ unsigned long long warp_sum36(unsigned long long x) {
  const uint32_t lo = __reduce_add_sync(0xffffffffu, (uint32_t)x & 0x3ffffu), hi = __reduce_add_sync(0xffffffffu, (uint32_t)(x >> 18));
  return lo + ((unsigned long long)hi << 18);
}
// Sum over the CTA, in every thread.
template <int kThreads>
__device__ __forceinline__ Tally block_sum(Shared& sm, Tally t) {
  t.mass = warp_sum(t.mass);
  t.count = __reduce_add_sync(0xffffffffu, t.count);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sm.red[threadIdx.x >> 5] = t;
  __syncthreads();
  t = {0ull, 0u};
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) t.mass += sm.red[i].mass, t.count += sm.red[i].count;
  return t;
}

__device__ __forceinline__ void hist_add_one(Shared& sm, bool on, uint32_t bin, uint32_t w) {
  if (!on) return;
  atomicAdd(&sm.hist[0][bin], 1u);
  atomicAdd(&sm.hist[1][bin], w & 0xffffu);
  atomicAdd(&sm.hist[2][bin], w >> 16);
}
// One element to the histogram (all lanes of the warp call it).  Lanes of one bin, as neighbours in id order are, add up first.
__device__ __forceinline__ void hist_add(Shared& sm, bool on, uint32_t bin, uint32_t w) {
  const unsigned mask = __ballot_sync(0xffffffffu, on);
  if (!mask) return;
  const uint32_t first = __shfl_sync(0xffffffffu, bin, __ffs(mask) - 1);
  if (__all_sync(0xffffffffu, !on || bin == first)) {
    const uint32_t lo = __reduce_add_sync(0xffffffffu, on ? w & 0xffffu : 0u), hi = __reduce_add_sync(0xffffffffu, on ? w >> 16 : 0u);
    if ((threadIdx.x & 31) == 0) {
      atomicAdd(&sm.hist[0][first], (uint32_t)__popc(mask));
      atomicAdd(&sm.hist[1][first], lo);
      atomicAdd(&sm.hist[2][first], hi);
    }
  } else {
    hist_add_one(sm, on, bin, w);
  }
}

// W of a logit: its quotient with T, the exponential of the difference from the maximum's, in the steps that define them.  Eight of
// a thread at a time, two an instruction, without branches.  The quotient is Markstein's (IBM J. Res. Dev. 34, 1990): from the
// correctly rounded 1 / T two corrections by the exact remainder give the correctly rounded quotient while nothing under- or
// overflows; in other rows (`plain` false) it is divided.  Rounding to a whole number is by adding 1.5 * 2^23, whose last bits then
// are that number.
struct Weigh {
  float temp, inverse, z_top;
  bool plain;
  __device__ __forceinline__ uint32_t operator()(float x) const {
    return __float2uint_rd(__fmul_rn(exp32_cw(__fsub_rn(__fdiv_rn(x, temp), z_top)), 2147483648.f));
  }
  __device__ __forceinline__ void eight(const float (&v)[8], uint32_t (&w)[8]) const {
    using namespace paged;
    auto both = [](float x) { return pack2(x, x); };
    uint64_t z[4];
    if (plain) {
      const uint64_t inv = both(inverse), minus = both(-temp);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // (-1e30 for -inf: W is 0 all the same)
        const uint64_t x = pack2(fmaxf(v[2 * e], -1e30f), fmaxf(v[2 * e + 1], -1e30f)), q0 = mul2(x, inv), q1 = fma2(fma2(q0, minus, x), inv, q0);
        z[e] = fma2(fma2(q1, minus, x), inv, q1);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = pack2(__fdiv_rn(v[2 * e], temp), __fdiv_rn(v[2 * e + 1], temp));
    }
    // (times one: ptxas makes a mul.rn.f32x2 and an add.rn.f32x2 that takes it one operation, rounded once)
    float alone = 1.f;
    asm("" : "+f"(alone));
    const uint64_t ones = both(alone);
    auto sum = [&](uint64_t a, uint64_t b) { return fma2(a, ones, b); };
    auto plus = [&](uint64_t a, float b) { return fma2(a, ones, both(b)); };
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float d[2], y[2], p[2];
      unpack2(add2(z[e], both(-z_top)), d[0], d[1]);
      const uint64_t x = pack2(fmaxf(d[0], -87.f), fmaxf(d[1], -87.f));
      const uint64_t t = plus(mul2(x, both(__int_as_float(0x3fb8aa3b))), 12582912.f), n = plus(t, -12582912.f);
      const uint64_t r = sum(sum(x, mul2(n, both(-__int_as_float(0x3f318000)))), mul2(n, both(-__int_as_float(0xb95e8083))));
      uint64_t s = both(__int_as_float(0x39500d01));
      s = plus(mul2(s, r), __int_as_float(0x3ab60b61));
      s = plus(mul2(s, r), __int_as_float(0x3c088889));
      s = plus(mul2(s, r), __int_as_float(0x3d2aaaab));
      s = plus(mul2(s, r), __int_as_float(0x3e2aaaab));
      s = plus(mul2(s, r), 0.5f);
      s = plus(mul2(s, r), 1.f);
      s = plus(mul2(s, r), 1.f);
      unpack2(t, y[0], y[1]);
      unpack2(s, p[0], p[1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {                    // (times 2^(n + 31): powers of two)
        // (from -87 down: 0, as the definition has it)
        w[2 * e + i] = __float2uint_rd(__fmul_rn(p[i], __uint_as_float((__float_as_uint(y[i]) << 23) + (158u << 23))));
      }
    }
  }
};

struct Level {
  uint32_t bin;
  Tally above, at;                     // of the bins above it, and of this one
};
// A histogram's sums, one bin a thread: thread t has bin 255 - t and what is above it.
struct Bins {
  Tally own, before;
};

// each(f) calls f(on, bin, w) for the CTA's elements, warp by warp.  With n > 1 the CTAs of the cluster count together, each its
// own elements, and have the same answer.
template <int kThreads, class Each>
__device__ __forceinline__ Bins count_bins(Shared& sm, int n, Tally above, Each each) {
  cg::cluster_group cl = cg::this_cluster();
  const int t = threadIdx.x, lane = t & 31;
  for (int i = t; i < 3 * 256; i += kThreads) (&sm.hist[0][0])[i] = 0u;
  __syncthreads();
  each([&](bool on, uint32_t bin, uint32_t w) { hist_add(sm, on, bin, w); });
  if (n > 1) cluster_sync();
  else __syncthreads();
  Bins b{{0ull, 0u}, above};
  if (t < 256) {
    uint32_t x[kMaxCluster][3];                        // (all on their way together: a turn each, they took 8,000 cycles)
#pragma unroll
    for (int z = 0; z < kMaxCluster; ++z) {
      const uint32_t* h = n > 1 ? cl.map_shared_rank(&sm.hist[0][0], min(z, n - 1)) : &sm.hist[0][0];
#pragma unroll
      for (int i = 0; i < 3; ++i) x[z][i] = z < n ? h[256 * i + 255 - t] : 0u;
    }
#pragma unroll
    for (int z = 0; z < kMaxCluster; ++z) b.own.count += x[z][0], b.own.mass += x[z][1] + ((unsigned long long)x[z][2] << 16);
    Tally run = b.own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned long long m = __shfl_up_sync(0xffffffffu, run.mass, d);
      const uint32_t c = __shfl_up_sync(0xffffffffu, run.count, d);
      if (lane >= d) run.mass += m, run.count += c;
    }
    if (lane == 31) sm.red[t >> 5] = run;
    b.before.mass += run.mass - b.own.mass, b.before.count += run.count - b.own.count;
  }
  // (others may still read: on every way from here a barrier of the cluster comes before a histogram is cleared or a CTA ends)
  __syncthreads();
  for (int i = 0; i < (t >> 5) && t < 256; ++i) b.before.mass += sm.red[i].mass, b.before.count += sm.red[i].count;
  return b;
}
// The bin at which the running sum (counts, or weights with by_mass) goes from below `target` to it or above.
__device__ __forceinline__ Level crossing(Shared& sm, const Bins& b, bool by_mass, unsigned long long target) {
  const unsigned long long x = by_mass ? b.before.mass : b.before.count, y = by_mass ? b.own.mass : b.own.count;
  __syncthreads();
  if (threadIdx.x < 256 && x < target && target - x <= y) sm.bin = 255 - threadIdx.x, sm.above = b.before, sm.at = b.own;
  __syncthreads();
  return {sm.bin, sm.above, sm.at};
}
// Sum of all bins.
__device__ __forceinline__ Tally bins_sum(Shared& sm, const Bins& b) {
  __syncthreads();
  if (threadIdx.x == 255) sm.at = {b.before.mass + b.own.mass, b.before.count + b.own.count};
  __syncthreads();
  return sm.at;
}

template <class T>
__device__ __forceinline__ float logit_at(const T* row, int i);
template <>
__device__ __forceinline__ float logit_at(const float* row, int i) { return __ldg(row + i); }
template <>
__device__ __forceinline__ float logit_at(const uint16_t* row, int i) { return bf16_bits_to_f32(__ldg(row + i)); }

// Eight logits as they lie.
template <class T>
struct Raw8;
template <>
struct Raw8<float> {
  static constexpr int kAhead = 2;
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4); }
  __device__ __forceinline__ void set(const float (&v)[8]) { a = make_float4(v[0], v[1], v[2], v[3]), b = make_float4(v[4], v[5], v[6], v[7]); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
};
template <>
struct Raw8<uint16_t> {
  static constexpr int kAhead = 4;
  uint4 a;
  __device__ __forceinline__ void load(const uint16_t* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    a = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo_f32(w[i]), v[2 * i + 1] = bf16_hi_f32(w[i]);
  }
};
// f(id, n, logits) for eight ids of a thread at a time, n of them in the share [lo, hi) (lo a multiple of 8), warp by warp: a
// warp's eights are 256 ids in a row.  The next ones are on their way while these are looked at.
template <class T, int kThreads, class F>
__device__ __forceinline__ void each_eight(const T* row, int lo, int hi, F f) {
  constexpr int kAhead = Raw8<T>::kAhead, kStep = kThreads * 8;
  const int lane = threadIdx.x & 31;
  int i = lo + (threadIdx.x & ~31) * 8;
  Raw8<T> next[kAhead];
  auto fetch = [&](int at, Raw8<T>& to) {
    const int c = at + lane * 8;
    if (c + 8 <= hi) {
      to.load(row + c);
    } else {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = c + e < hi ? logit_at(row, c + e) : 0.f;
      to.set(v);
    }
  };
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (i + k * kStep < hi) fetch(i + k * kStep, next[k]);
#pragma unroll 1
  for (; i < hi; i += kStep) {
    float v[8];
    next[0].get(v);
#pragma unroll
    for (int k = 0; k + 1 < kAhead; ++k) next[k] = next[k + 1];
    if (i + kAhead * kStep < hi) fetch(i + kAhead * kStep, next[kAhead - 1]);
    f(i + lane * 8, min(8, hi - i - lane * 8), v);
  }
}

// kAlone: a CTA a row.  (Without the cluster's code 128 rows of 2,048 take 14.7 us and 1,000 take 29; with it 16.2 and 34.
// Four CTAs an SM of 64 registers a thread instead of three of 80: 400 rows of 131,072 take 143 us instead of 164; 128 of 2,048, which
// all run at a time, 13.2 instead of 12.5.)
template <class T, bool kAlone, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads > 256 ? 1 : kAlone ? 3 : kPerSm) sample_kernel(const SampleArgs a) {
  __shared__ Shared shared;
  Shared& sm = shared;
  constexpr int kWarps = kThreads / 32;
  static_assert(kThreads >= 256 && kWarps <= kMaxWarps, "a thread a bin");
  cg::cluster_group cl = cg::this_cluster();
  const int n = kAlone ? 1 : a.cluster, rank = n > 1 ? (int)cl.block_rank() : 0, t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int V = a.vocab, per = ((V + n - 1) / n + 7) / 8 * 8, lo = min(V, rank * per), hi = min(V, lo + per);
  auto meet = [&] {
    if (n > 1) cluster_sync();
    else __syncthreads();
  };
  if (n > 1) cluster_arrive();
  tc::pdl_wait();
  tc::pdl_trigger();
  long long r = blockIdx.x / n;
  if (!kAlone && a.ordered) {                          // of 256 rows: weighed ones, then those of a list, then greedy ones
    const long long from = r & ~255ll;
    const bool on = t < 256 && from + t < a.n_rows;
    int kind = 3;
    if (on) {
      const float p = a.top_p ? __ldg(a.top_p + from + t) : 1.f;
      const int k = a.top_k ? __ldg(a.top_k + from + t) : 0;
      kind = (a.temperature && __ldg(a.temperature + from + t) == 0.f) || k == 1 || p <= 0.f ? 2 : p < 1.f && (k <= 0 || k > kMostGroups) ? 0 : 1;
    }
    uint32_t at = 0u;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const unsigned same = __ballot_sync(0xffffffffu, kind == i);
      if (lane == 0) sm.kinds[i][warp] = __popc(same);
      if (kind == i) at = __popc(same & ((1u << lane) - 1u));
    }
    __syncthreads();
    if (on) {
      for (int i = 0; i <= kind; ++i)
        for (int w = 0; w < (i < kind ? kWarps : warp); ++w) at += sm.kinds[i][w];
      if (from + at == r) sm.row = (uint32_t)t;
    }
    __syncthreads();
    r = from + sm.row;
  }
  const T* row = static_cast<const T*>(a.logits) + r * a.stride;
  const float temp = a.temperature ? __ldg(a.temperature + r) : 1.f, top_p = a.top_p ? __ldg(a.top_p + r) : 1.f,
              min_p = a.min_p ? __ldg(a.min_p + r) : 0.f;
  const int top_k = a.top_k ? __ldg(a.top_k + r) : 0;
  const double u = __ldg(a.u + r);

  // ---- the largest logit
  Told mine = {};
  {
    float most = -INFINITY;
    bool bad = false, odd = false;
    each_eight<T, kThreads>(row, lo, hi, [&](int, int left, const float (&v)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e >= left) continue;
        most = fmaxf(most, v[e]);
        bad |= !(v[e] <= 3.40282347e38f);              // NaN or +inf
        const uint32_t size = __float_as_uint(v[e]) & 0x7fffffffu;      // 2^-99 .. 2^95, 0 or -inf
        odd |= size - 0x0e000000u >= 0x61000000u && size != 0u && size != 0x7f800000u;
      }
    });
    // (as few groups as there must be: a list of k ln k ids, about)
    int group = 32;
    while (group > 1 && n * (kThreads / group) < top_k && n * (kThreads / group) < kMostGroups) group /= 2;
    for (int w = group / 2; w; w >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, w));
    const uint32_t key = key_of(most);
    const float warp_top = logit_of(__reduce_max_sync(0xffffffffu, key)), warp_least = logit_of(__reduce_min_sync(0xffffffffu, key));
    const int flags = (int)__any_sync(0xffffffffu, bad) | (int)__any_sync(0xffffffffu, odd) << 1;
    if (lane == 0) sm.fred[0][warp] = warp_top, sm.fred[1][warp] = warp_least, sm.flags[warp] = flags;
    __syncthreads();
    mine.top = -INFINITY, mine.least = INFINITY;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      mine.top = fmaxf(mine.top, sm.fred[0][i]), mine.least = fminf(mine.least, sm.fred[1][i]);
      mine.bad |= sm.flags[i] & 1, mine.odd |= sm.flags[i] >> 1;
    }
  }
  // (every CTA's `mine` to all)
  auto tell = [&](int what) {
    if (t < n) *(n > 1 ? cl.map_shared_rank(&sm.told[what][rank], t) : &sm.told[what][0]) = mine;
    meet();
  };
  if (n > 1) cluster_wait();                        // (the others have started)
  tell(0);
  float top = -INFINITY, least = INFINITY;
  bool plain = temp > 1e-6f && temp < 1e6f;
  bool bad = !(temp >= 0.f && temp <= 3.40282347e38f) || isnan(top_p) || isnan(min_p) || !(u >= 0. && u < 1.);
  for (int z = 0; z < n; ++z) top = fmaxf(top, sm.told[0][z].top), least = fminf(least, sm.told[0][z].least), bad |= sm.told[0][z].bad != 0, plain &= sm.told[0][z].odd == 0;
  bad |= top == -INFINITY;
  auto give = [&](uint32_t id, unsigned long long w, Tally in) {
    a.ids[r] = (int)id;
    if (a.probs) a.probs[r] = (float)((double)w / (double)in.mass);
    if (a.kept) a.kept[r] = (int)in.count;
  };
  if (bad) {                                           // (every CTA of the cluster alike, here and below)
    if (rank == 0 && t == 0) {
      atomicCAS(a.err, 0, (int)MCD_ERR_INVALID_ARG);
      give(0xffffffffu, 0ull, {1ull, 0u});
    }
    return;
  }
  const uint32_t key_top = key_of(top);
  const float z_top = __fdiv_rn(top, temp);
  const bool has_p = top_p < 1.f;
  bool has_k = top_k > 0 && top_k < V;
  const bool greedy = temp == 0.f || !(fabsf(z_top) <= 3.40282347e38f) || top_k == 1 || top_p <= 0.f;
  const uint32_t w_min = min_p > 0.f ? max(1u, (uint32_t)ceil((double)fminf(min_p, 1.f) * 2147483648.)) : 1u;
  const Weigh weight{temp, __fdiv_rn(1.f, temp), z_top, plain && fabsf(top) < 1e28f};
  // no id below it has a weight that counts (the margins cover the roundings of quotient, difference and exponential)
  const float floor_x = top + temp * fmaxf(-22.f, w_min > 1u ? logf(fminf(min_p, 1.f)) - 1e-3f : -22.f) - fabsf(top) * 1e-6f;

  bool listed = false;
  // f(on, key, id, weigh) for the CTA's share of the row, or (the first CTA alone) of the list, warp by warp
  auto each = [&](auto f) {
    if (listed) {
      const int count = min((int)sm.n_list, kList);
      for (int i = t & ~31; i < count; i += kThreads) {
        const int j = min(i + lane, count - 1);
        f(i + lane < count && sm.w[j] > 0u, sm.key[j], sm.id[j], [&] { return sm.w[j]; });
      }
    } else {
      each_eight<T, kThreads>(row, lo, hi, [&](int id, int left, const float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = v[e];
          f(e < left, key_of(x), (uint32_t)(id + e), [&] { return weight(x); });
        }
      });
    }
  };
  // the least and largest of what `of` gives where it is not ~0
  auto extent = [&](auto of) {
    uint32_t from = 0xffffffffu, to = 0u;
    each([&](bool on, uint32_t key, uint32_t id, auto) {
      const uint32_t x = on ? of(key, id) : 0xffffffffu;
      if (x != 0xffffffffu) from = min(from, x), to = max(to, x);
    });
    from = __reduce_min_sync(0xffffffffu, from), to = __reduce_max_sync(0xffffffffu, to);
    __syncthreads();
    if (lane == 0) sm.ured[0][warp] = from, sm.ured[1][warp] = to;
    __syncthreads();
    for (int i = 0; i < kWarps; ++i) from = min(from, sm.ured[0][i]), to = max(to, sm.ured[1][i]);
    if (!listed && n > 1) {
      mine.lo = from, mine.hi = to;
      tell(2);
      for (int z = 0; z < n; ++z) from = min(from, sm.told[2][z].lo), to = max(to, sm.told[2][z].hi);
      meet();
    }
    return make_uint2(from, to);
  };
  if (greedy) {
    const uint2 at = extent([&](uint32_t key, uint32_t id) { return key == key_top ? id : 0xffffffffu; });
    if (rank == 0 && t == 0) give(at.x, 1ull, {1ull, 1u});
    return;
  }
  // the CTAs' lists, if the first one's holds them all, to it; how many ids they have
  auto together = [&] {
    if (n == 1) return sm.n_list;
    mine.lo = sm.n_list;
    tell(3);
    uint32_t sum = 0u;
    for (int z = 0; z < n; ++z) sum += sm.told[3][z].lo;
    if (sum <= (uint32_t)kList) {
      if (rank > 0) {
        uint32_t from = 0u;
        for (int z = 0; z < rank; ++z) from += sm.told[3][z].lo;
        Shared& first = *cl.map_shared_rank(&sm, 0);
        for (uint32_t i = t; i < mine.lo; i += kThreads) first.key[from + i] = sm.key[i], first.id[from + i] = sm.id[i], first.w[from + i] = sm.w[i];
      } else if (t == 0) {
        sm.n_list = sum;
      }
    }
    cluster_sync();                                         // (the lists have come)
    return sum;
  };
  // the row's ids that `want` takes (weighed: those of them with weight): to each CTA's list, and if there are no more than it holds, all to the
  // first one's; how many there are
  auto gather = [&](bool weighed, auto want) {
    if (t == 0) sm.n_list = 0u;
    __syncthreads();
    each_eight<T, kThreads>(row, lo, hi, [&](int id, int left, const float (&v)[8]) {
      uint32_t on = 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e) on |= (uint32_t)(e < left && want(v[e])) << e;
      if (weighed && __any_sync(0xffffffffu, on != 0u)) {
        uint32_t w[8];
        weight.eight(v, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) on &= ~((uint32_t)(w[e] == 0u) << e);
      }
      // (few of a warp's ids, as a rule: one of a lane at a time)
      for (unsigned mask; (mask = __ballot_sync(0xffffffffu, on != 0u)) != 0u; on &= on - 1u) {
        uint32_t at = 0u;
        if (lane == 0) at = atomicAdd(&sm.n_list, (uint32_t)__popc(mask));
        at = __shfl_sync(0xffffffffu, at, 0) + __popc(mask & ((1u << lane) - 1u));
        const int first = __ffs(on) - 1;
        float x = v[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) x = e == first ? v[e] : x;
        if (on != 0u && at < (uint32_t)kList) sm.key[at] = key_of(x), sm.id[at] = (uint32_t)(id + first);
      }
    });
    __syncthreads();
    // their weights
    const int count = min((int)sm.n_list, kList);
    for (int i = t * 8; i < count; i += kThreads * 8) {
      float v[8];
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = i + e < count ? logit_of(sm.key[i + e]) : 0.f;
      weight.eight(v, w);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i + e < count) sm.w[i + e] = w[e];
    }
    __syncthreads();
    return together();
  };
  // narrows [at.x, at.y], a range of what `of` gives, to the one value where the running sum over descending values reaches the
  // target; in: its sums, as far as they are known
  auto narrow = [&](uint2 at, bool by_mass, unsigned long long target, Tally above, Tally in, uint32_t least_w, auto of) {
    Level l{0u, above, in};
    for (int rounds = 0; at.x != at.y; ++rounds) {
      if (rounds > 4 || at.x > at.y) {                 // (eight bits a round; a set without the target would be a fault of this kernel)
        if (rank == 0 && t == 0) atomicCAS(a.err, 0, (int)MCD_ERR_TIMEOUT);
        break;
      }
      const int bits = 32 - __clz(at.y - at.x), shift = bits > 8 ? bits - 8 : 0;
      const Bins b = count_bins<kThreads>(sm, listed ? 1 : n, l.above, [&](auto add) {
        each([&](bool on, uint32_t key, uint32_t id, auto weigh) {
          const uint32_t x = on ? of(key, id) : 0xffffffffu;
          on = x != 0xffffffffu && x >= at.x && x <= at.y;
          const uint32_t w = on ? weigh() : 0u;
          add(on && w >= least_w, on ? (x - at.x) >> shift : 0u, w);
        });
      });
      l = crossing(sm, b, by_mass, target);
      const uint32_t from = at.x + (l.bin << shift), to = from + min(at.y - from, (1u << shift) - 1u);
      at = from == to ? make_uint2(from, to) : extent([&](uint32_t key, uint32_t id) {
        const uint32_t x = of(key, id);
        return x >= from && x <= to ? x : 0xffffffffu;
      });
    }
    l.bin = at.x;
    return l;
  };
  auto from_id = [V](uint32_t id) { return (uint32_t)(V - 1) - id; };

  // ---- cuts
  Cut cut{0x007fffffu, 0xffffffffu, {0ull, 0u}};       // (the key of -inf: nothing is cut)
  auto logit_before_cut = [&](float x, uint32_t id) {
    const float c = logit_of(cut.key);
    return x > c || (x == c && id <= cut.id);
  };
  auto before_cut = [&](uint32_t key, uint32_t id) { return key > cut.key || (key == cut.key && id <= cut.id); };
  // steps of the histograms: from the maximum down to where W is 0 (2^31 e^-21.5 < 1), or to the list's end.  (22 T would leave fp32's
  // range from 1.5e37 on, and 0 times -inf's distance, NaN, put hidden ids beside the maximum; a tiny T's quotient leaves it too)
  float scale = fminf(255.f / 22.f / temp, 3.40282347e38f);
  auto bin_of = [&](float x) { return 255u - (uint32_t)min(255, (int)((top - x) * scale)); };
  auto key_bins = [&] {
    return count_bins<kThreads>(sm, listed ? 1 : n, {0ull, 0u}, [&](auto) {
      if (listed) {
        each([&](bool on, uint32_t key, uint32_t id, auto weigh) {
          hist_add_one(sm, on && before_cut(key, id), bin_of(logit_of(key)), weigh());
        });
      } else {
        each_eight<T, kThreads>(row, lo, hi, [&](int, int left, const float (&v)[8]) {
          uint32_t w[8];
          weight.eight(v, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) hist_add_one(sm, e < left && w[e] > 0u, bin_of(v[e]), w[e]);
        });
      }
    });
  };
  // the few ids that `want` takes, to the short list
  auto gather_few = [&](auto want) {
    if (t == 0) sm.n_few = 0u;
    __syncthreads();
    each([&](bool on, uint32_t key, uint32_t id, auto weigh) {
      on = on && want(key, id, weigh());
      const unsigned mask = __ballot_sync(0xffffffffu, on);
      if (!mask) return;
      uint32_t at = 0u;
      if (lane == 0) at = atomicAdd(&sm.n_few, (uint32_t)__popc(mask));
      at = __shfl_sync(0xffffffffu, at, 0) + __popc(mask & ((1u << lane) - 1u));
      if (on && at < (uint32_t)kFew) sm.few[at] = make_uint4(key, id, weigh(), 0u);
    });
    __syncthreads();
    return min((int)sm.n_few, kFew);
  };
  // the cut in bin l.bin
  auto cut_in = [&](const Level coarse, bool by_mass, unsigned long long target) {
    const Cut old = cut;
    Level l = coarse;
    bool fine = false;
    auto part_of = [&](float x) { return 255u - (uint32_t)min(255, max(0, (int)(__fsub_rn(__fmul_rn(top - x, scale), (float)(255u - coarse.bin)) * 256.f))); };
    auto member = [&](uint32_t key, uint32_t id) {
      const float x = logit_of(key);
      return (key > old.key || (key == old.key && id <= old.id)) && bin_of(x) == coarse.bin && (!fine || part_of(x) == l.bin);
    };
    if (listed && l.at.count > (uint32_t)kFew) {       // 256 parts of the bin
      const Bins b = count_bins<kThreads>(sm, 1, coarse.above, [&](auto) {
        each([&](bool on, uint32_t key, uint32_t id, auto weigh) { hist_add_one(sm, on && member(key, id), part_of(logit_of(key)), weigh()); });
      });
      l = crossing(sm, b, by_mass, target);
      fine = true;
    }
    if (listed && l.at.count <= (uint32_t)kFew) {
      const int few = gather_few([&](uint32_t key, uint32_t id, uint32_t) { return member(key, id); });
      if (t < few) {
        const uint4 me = sm.few[t];
        const uint32_t key = me.x, id = me.y, w = me.z;
        Tally b = l.above;
#pragma unroll 8
        for (int j = 0; j < few; ++j) {
          const uint4 o = sm.few[j];
          const bool first = (o.x > key) | ((o.x == key) & (o.y < id));
          b.mass += first ? o.z : 0u, b.count += first;
        }
        const unsigned long long x = by_mass ? b.mass : b.count;
        if (x < target && target - x <= (by_mass ? w : 1u)) sm.cut = {key, id, {b.mass + w, b.count + 1u}};
      }
      __syncthreads();
      cut = sm.cut;
      __syncthreads();
      return;
    }
    auto of = [&](uint32_t key, uint32_t id) { return member(key, id) ? key : 0xffffffffu; };
    const Level p = narrow(extent(of), by_mass, target, l.above, l.at, 1u, of);
    // (p.at can hold ids behind the old cut: it does not tell the weight, and of the count only that there are no more)
    const unsigned long long one = weight(logit_of(p.bin));
    const uint32_t ties = (uint32_t)(by_mass ? (target - p.above.mass + one - 1) / one : target - p.above.count);
    cut.key = p.bin;
    if (ties < p.at.count) {
      auto tie = [&](uint32_t key, uint32_t id) { return key == cut.key && (key > old.key || id <= old.id) ? from_id(id) : 0xffffffffu; };
      if (listed && p.at.count <= (uint32_t)kFew) {
        const int few = gather_few([&](uint32_t key, uint32_t id, uint32_t) { return tie(key, id) != 0xffffffffu; });
        if (t < few) {
          const uint32_t id = sm.few[t].y;
          uint32_t before = 0u;
          for (int j = 0; j < few; ++j) before += sm.few[j].y < id;
          if (before == ties - 1u) sm.cut.id = id;
        }
        __syncthreads();
        cut.id = sm.cut.id;
        __syncthreads();
      } else {
        cut.id = from_id(narrow(extent(tie), false, ties, {0ull, 0u}, {0ull, 0u}, 1u, tie).bin);
      }
    } else if (cut.key > old.key) {
      cut.id = 0xffffffffu;
    }
    cut.in = {p.above.mass + one * ties, p.above.count + ties};
  };
  // (top_p < 1 and a mass below 2^50: the product is at most the mass)
  auto need_of = [&](unsigned long long mass) { return min(max(1ull, (unsigned long long)ceil((double)top_p * (double)mass)), mass); };

  // Sums of W, of blocks of 256 ids and of all, of the row's ids before the cut; or, with a cut that is still to be found in bin l.bin,
  // of those in the bins above, while that one's ids go to the CTA's list.
  Tally sums{0ull, 0u};
  auto sum_row = [&](auto is_open, uint32_t bin) {
    constexpr bool open = decltype(is_open)::value;
    if (t == 0) sm.n_list = 0u;
    __syncthreads();
    const float from = fmaxf(floor_x, logit_of(cut.key));
    sums = {0ull, 0u};
    int i = warp;
    each_eight<T, kThreads>(row, lo, hi, [&](int id, int left, const float (&v)[8]) {
      Tally y{0ull, 0u};
      float most = v[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) most = fmaxf(most, v[e]);
      if (__any_sync(0xffffffffu, open ? bin_of(most) >= bin : most >= from)) {
        uint32_t w[8], on = 0u;
        weight.eight(v, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          bool in = e < left && w[e] >= w_min;
          if constexpr (open) {
            const uint32_t b = bin_of(v[e]);
            on |= (uint32_t)(e < left && w[e] > 0u && b == bin) << e;
            in = in && b > bin;
          } else {
            in = in && logit_before_cut(v[e], (uint32_t)(id + e));
          }
          y.mass += in ? w[e] : 0u, y.count += in;
        }
        y.mass = warp_sum36(y.mass);                   // (eight of 2^31 at most)
        if constexpr (open) {
          for (unsigned mask; (mask = __ballot_sync(0xffffffffu, on != 0u)) != 0u; on &= on - 1u) {
            uint32_t at = 0u;
            if (lane == 0) at = atomicAdd(&sm.n_list, (uint32_t)__popc(mask));
            at = __shfl_sync(0xffffffffu, at, 0) + __popc(mask & ((1u << lane) - 1u));
            const int first = __ffs(on) - 1;
            float x = v[0];
            uint32_t own = w[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) x = e == first ? v[e] : x, own = e == first ? w[e] : own;
            if (on != 0u && at < (uint32_t)kList) sm.key[at] = key_of(x), sm.id[at] = (uint32_t)(id + first), sm.w[at] = own;
          }
        }
      }
      if (lane == 0) sm.block[i] = y.mass, sums.mass += y.mass;
      sums.count += y.count;
      i += kWarps;
    });
    __syncthreads();
  };

  bool p_done = false, summed = false;
  if (has_k && top_k <= kMostGroups) {
    // a rounded quotient can put an id of weight below the point where none should have any: 1e-6 of the logits covers it
    const float near = fmaxf(least, top - 22.f * temp - fabsf(top) * 1e-6f);
    listed = gather(false, [&](float x) { return x >= near; }) <= (uint32_t)kList;
    if (listed) {
      if (rank > 0) return;
      const float span = top - near;
      scale = span > 0.f ? fminf(255.f / span, 3.40282347e38f) : 0.f;
      const Bins b = key_bins();
      cut.in = bins_sum(sm, b);
      if ((uint32_t)top_k < cut.in.count) cut_in(crossing(sm, b, false, top_k), false, top_k);
    }
  }
  if ((has_k || has_p) && !listed) {
    const Bins b = key_bins();
    cut.in = bins_sum(sm, b);
    has_k = has_k && (uint32_t)top_k < cut.in.count;
    unsigned long long target = has_k ? (unsigned long long)top_k : need_of(cut.in.mass);
    // (a bin's ids to the list, or all down to it: the first CTA alone finds the cut and, in the first case, tells the others)
    auto find = [&](const Level l, bool by_mass, bool last) {
      if (last && w_min > 1u && bin_of(floor_x) > l.bin) return;      // (min_p leaves less than the cut)
      const bool all = l.above.count + l.at.count <= (uint32_t)kList;
      // (the bins have counted ids of weight alone; the last ones, and all where a difference of quotients is coarse, hold others
      // too, which could be too many: so can all of a T below 3e-38, whose first bin is wider than what has weight)
      uint32_t own = 0u, held = kList + 1;
      if (all || l.at.count <= (uint32_t)kList) {
        if (!all && last) {
          sum_row(std::true_type{}, l.bin);
          own = sm.n_list;
          held = together();
          summed = true;
        } else {
          held = gather(l.bin < 16u || fabsf(z_top) > 1e4f, [&](float x) { return all ? bin_of(x) >= l.bin : bin_of(x) == l.bin; });
        }
      }
      if (held > (uint32_t)kList) {                    // (no list, or it has not come together: from the row)
        summed = false;
        cut_in(l, by_mass, target);
        return;
      }
      listed = all;
      if (rank > 0 && all) return;
      if (rank == 0) {
        listed = true;
        cut_in(l, by_mass, target);
        listed = all;
      }
      if (all) return;
      if (rank == 0) {
        if (t < n) *(n > 1 ? cl.map_shared_rank(&sm.cut, t) : &sm.cut) = cut;
      }
      meet();
      cut = sm.cut;
      if (summed) {
        for (uint32_t i = t; i < own; i += kThreads) {
          const uint32_t w = sm.w[i];
          if (w >= w_min && before_cut(sm.key[i], sm.id[i])) {
            atomicAdd(&sm.block[(sm.id[i] - (uint32_t)lo) >> 8], (unsigned long long)w);
            sums.mass += w, ++sums.count;
          }
        }
      }
    };
    if (has_k || has_p) {
      find(crossing(sm, b, !has_k, target), !has_k, !(has_k && has_p));
      if (listed && rank > 0) return;
      p_done = !has_k;
      if (has_k && has_p && !listed) {
        target = need_of(cut.in.mass);
        find(crossing(sm, b, true, target), true, true);
        if (listed && rank > 0) return;
        p_done = true;
      }
    }
  }

  // ---- the draw
  if (!listed) {
    if (!summed) sum_row(std::false_type{}, 0u);
    mine.sum = block_sum<kThreads>(sm, sums);
    tell(1);
    Tally in{0ull, 0u};
    unsigned long long ahead = 0ull;
    for (int z = 0; z < n; ++z) {
      if (z < rank) ahead += sm.told[1][z].sum.mass;
      in.mass += sm.told[1][z].sum.mass, in.count += sm.told[1][z].sum.count;
    }
    const unsigned long long drawn = min((unsigned long long)floor(u * (double)in.mass), in.mass - 1);
    if (drawn < ahead || drawn - ahead >= mine.sum.mass || warp > 0) return;
    unsigned long long rest = drawn - ahead;           // (in this CTA's share)
    const int blocks = (hi - lo + 255) / 256;
    int from = 0;
    for (; from < blocks; from += 32) {                // the block, 32 at a time
      const unsigned long long own = from + lane < blocks ? sm.block[from + lane] : 0ull;
      unsigned long long run = own;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xffffffffu, run, d);
        if (lane >= d) run += y;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, rest < run);
      if (hit) {
        const int f = __ffs(hit) - 1;
        rest -= __shfl_sync(0xffffffffu, run - own, f);
        from += f;
        break;
      }
      rest -= __shfl_sync(0xffffffffu, run, 31);
    }
    const int id = lo + from * 256 + lane * 8;
    uint32_t w[8];
    unsigned long long own = 0ull;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = 0u;
      if (id + e >= hi) continue;
      const float x = logit_at(row, id + e);
      if (before_cut(key_of(x), (uint32_t)(id + e))) w[e] = weight(x);
      if (w[e] < w_min) w[e] = 0u;
      own += w[e];
    }
    unsigned long long run = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned long long y = __shfl_up_sync(0xffffffffu, run, d);
      if (lane >= d) run += y;
    }
    unsigned long long at = run - own;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (w[e] > 0u && at <= rest && rest < at + w[e]) give((uint32_t)(id + e), w[e], in);
      at += w[e];
    }
    return;
  }
  // from the list (the first CTA alone)
  if (has_p && !p_done && cut.in.count > (uint32_t)kFew) {
    const unsigned long long need = need_of(cut.in.mass);
    const Bins b = key_bins();
    cut_in(crossing(sm, b, true, need), true, need);
    p_done = true;
  }
  if (cut.in.count <= (uint32_t)kFew) {
    const int few = gather_few([&](uint32_t key, uint32_t id, uint32_t) { return before_cut(key, id); });
    const unsigned long long need = has_p && !p_done ? need_of(cut.in.mass) : ~0ull;
    uint32_t key = 0u, id = 0u, w = 0u;
    if (t < few) {
      const uint4 me = sm.few[t];
      key = me.x, id = me.y, w = me.z;
      unsigned long long b = 0ull;
      if (need != ~0ull) {
#pragma unroll 8
        for (int j = 0; j < few; ++j) {
          const uint4 o = sm.few[j];
          b += (o.x > key) | ((o.x == key) & (o.y < id)) ? o.z : 0u;
        }
      }
      if (b >= need || w < w_min) w = 0u;
    }
    __syncthreads();
    if (t < few) sm.few[t].z = w;
    const Tally in = block_sum<kThreads>(sm, {w, w > 0u});
    const unsigned long long drawn = min((unsigned long long)floor(u * (double)in.mass), in.mass - 1);
    if (w > 0u) {
      unsigned long long b = 0ull;
#pragma unroll 8
      for (int j = 0; j < few; ++j) {
        const uint4 o = sm.few[j];
        b += o.y < id ? o.z : 0u;
      }
      if (b <= drawn && drawn < b + w) give(id, w, in);
    }
    return;
  }
  // (256 parts of the ids, and the few of one, as a rule)
  const int part = max(0, 24 - __clz(V - 1));
  const Bins b = count_bins<kThreads>(sm, 1, {0ull, 0u}, [&](auto) {
    each([&](bool on, uint32_t key, uint32_t id, auto weigh) {
      const uint32_t w = weigh();
      hist_add_one(sm, on && w >= w_min && before_cut(key, id), 255u - (id >> part), w);
    });
  });
  const Tally in = bins_sum(sm, b);
  const unsigned long long drawn = min((unsigned long long)floor(u * (double)in.mass), in.mass - 1);
  const Level l = crossing(sm, b, true, drawn + 1);
  if (l.at.count <= (uint32_t)kFew) {
    const int few = gather_few([&](uint32_t key, uint32_t id, uint32_t w) { return w >= w_min && 255u - (id >> part) == l.bin && before_cut(key, id); });
    if (t < few) {
      const uint32_t id = sm.few[t].y, w = sm.few[t].z;
      unsigned long long before = l.above.mass;
#pragma unroll 8
      for (int j = 0; j < few; ++j) {
        const uint4 o = sm.few[j];
        before += o.y < id ? o.z : 0u;
      }
      if (before <= drawn && drawn < before + w) give(id, w, in);
    }
    return;
  }
  auto of = [&](uint32_t key, uint32_t id) { return before_cut(key, id) ? from_id(id) : 0xffffffffu; };
  const Level p = narrow(extent(of), true, drawn + 1, {0ull, 0u}, in, w_min, of);
  if (t == 0) give(from_id(p.bin), p.at.mass, in);
}

// CTAs of a row: enough that each has 8,192 ids at most; 4,096 where there are so few rows that all have SMs of their own (8 rows of
// 16,384, top_p 0.9: 17.9 -> 15.6 us, k = 50 11.8 -> 10.4; 1,000 rows of 32,768 would take 197 us instead of 129).
int cluster_for(int vocab, long long n_rows) {
  int n = 1;
  while (n < kMaxCluster && (vocab > n * 8192 || (vocab > n * 4096 && n_rows * 2 * n <= paged::sm_count()))) n *= 2;
  return n;
}

}  // namespace

template <class T>
cudaError_t launch_sample(SampleArgs a, int n_rows, cudaStream_t st) {
  a.cluster = cluster_for(a.vocab, n_rows);
  a.n_rows = n_rows;
  // Rows that wait for SMs: those that take 45 us go first, those of 20 fill the ends (96 rows of 131,072: 52 us against 68 in their
  // own order; 400: 173 against 195, measured with three CTAs an SM).  Where all run at a time it would only cost the look at the settings.
  a.ordered = (long long)n_rows * a.cluster > kPerSm * paged::sm_count();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n_rows * a.cluster);
  const bool wide = (long long)n_rows * a.cluster <= paged::sm_count();
  cfg.blockDim = dim3(a.cluster > 1 && wide ? 512 : 256);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = a.cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  auto* kernel = a.cluster == 1 ? sample_kernel<T, true, 256> : wide ? sample_kernel<T, false, 512> : sample_kernel<T, false, 256>;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace rows
}  // namespace mcd
