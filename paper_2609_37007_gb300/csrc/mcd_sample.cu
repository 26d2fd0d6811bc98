// mcd_sample_rows (include/mcd_rows.h): one id of every logits row by temperature, top-k, top-p and min-p.
//
// The mathematics is in whole numbers: an id's weight is W = floor(2^31 exp32(logit / T - z_max)), and every filter is a cut of the
// ranking (logit descending, id ascending): "the first k", "until the weights' sum reaches a target", "no weight below".
// A cut is found without sorting, by a radix selection: a histogram (counts and sums of W) of the leading 8 bits of what is
// left of the keys' range, the bin in which the target is crossed, then the next 8 bits in that bin.  The draw is the same
// selection on ids in ascending order, its target a sum of weights.
//
// A cluster of CTAs takes a row.  It reads it for the maximum and, from the caches, once more: then ids within kNear of the
// maximum (in units of T) go to a list in the first CTA's shared memory, and the sum of all weights is formed where top_p wants
// it.  The list usually holds every id that the cuts leave, and the first CTA goes on alone with it; where it does not (or
// nothing is cut), the whole cluster makes the selections' histograms from the row itself.
// Order never changes a result: whole numbers add up to the same sum.
#include <cooperative_groups.h>

#include <cmath>

#include "mcd_rows.cuh"
#include "mcd_sampler.cuh"

namespace mcd {
namespace rows {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;
constexpr int kMaxCluster = 8;
constexpr int kList = 3584;            // ids of the list
constexpr float kNear = 8.f;
constexpr int kMaxVocabRows = 1 << 18;

struct SampleArgs {
  const void* logits;
  long long stride;
  int vocab, cluster;
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  const double* u;
  int32_t* ids;
  float* probs;
  int32_t* kept;
  int32_t* err;
};

// Keys in the order of the logits (finite ones and -inf): a larger logit has a larger key; -0 is 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct Tally {
  unsigned long long mass;
  uint32_t count;
};
// What a CTA tells the others.
struct Told {
  float top;
  int bad;
  Tally all, near;
};

struct Shared {
  uint32_t hist[3][256];               // counts, sums of the low 16 bits of W, of the others
  uint32_t key[kList], id[kList], w[kList];
  uint32_t n_list;
  Told told[3][kMaxCluster];           // of the maximum, of the lists, of the cuts
  Tally red[kThreads / 32];
  float fred[kThreads / 32];
  uint32_t bin;
  Tally above, at;
};

__device__ __forceinline__ unsigned long long warp_sum(unsigned long long x) {
#pragma unroll
  for (int w = 16; w; w >>= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
  return x;
}
// Sum over the CTA, in every thread.
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
  } else if (on) {
    atomicAdd(&sm.hist[0][bin], 1u);
    atomicAdd(&sm.hist[1][bin], w & 0xffffu);
    atomicAdd(&sm.hist[2][bin], w >> 16);
  }
}

struct Pick {
  uint32_t key;
  Tally above, at;                     // of the larger keys, and of this one
};

// The largest key at which the running sum over descending keys (counts, or weights with by_mass) reaches `target` (at
// least 1, at most the whole sum).  Keys are in [lo, lo + 2^bits); each(f) calls f(on, key, w) for the CTA's elements, warp by
// warp.  With n > 1 the CTAs of the cluster do it together, each with its own elements.
template <class Each>
__device__ __forceinline__ Pick pick(Shared& sm, int n, uint32_t lo, int bits, bool by_mass, unsigned long long target, Each each) {
  cg::cluster_group cl = cg::this_cluster();
  const int t = threadIdx.x;
  Pick p{lo, {0ull, 0u}, {0ull, 0u}};
  do {
    const int shift = bits > 8 ? bits - 8 : 0;
    for (int i = t; i < 3 * 256; i += kThreads) (&sm.hist[0][0])[i] = 0u;
    __syncthreads();
    const uint32_t base = p.key;
    each([&](bool on, uint32_t key, uint32_t w) {
      const uint32_t r = key - base;
      on = on && key >= base && (bits >= 32 || r >> bits == 0);
      hist_add(sm, on, on ? r >> shift : 0u, w);
    });
    if (n > 1) cl.sync();
    else __syncthreads();
    // bins in descending order, one a thread
    Tally own{0ull, 0u};
    if (t < 256) {
      const int b = 255 - t;
      for (int z = 0; z < n; ++z) {
        const uint32_t* h = n > 1 ? cl.map_shared_rank(&sm.hist[0][0], z) : &sm.hist[0][0];
        own.count += h[b];
        own.mass += h[256 + b] + ((unsigned long long)h[512 + b] << 16);
      }
    }
    Tally run = own;
    const int lane = t & 31;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned long long m = __shfl_up_sync(0xffffffffu, run.mass, d);
      const uint32_t c = __shfl_up_sync(0xffffffffu, run.count, d);
      if (lane >= d) run.mass += m, run.count += c;
    }
    if (t < 256 && lane == 31) sm.red[t >> 5] = run;
    __syncthreads();
    if (t < 256) {
      Tally from = p.above;
      for (int i = 0; i < t >> 5; ++i) from.mass += sm.red[i].mass, from.count += sm.red[i].count;
      const Tally before{from.mass + run.mass - own.mass, from.count + run.count - own.count};
      const unsigned long long x = by_mass ? before.mass : before.count, y = by_mass ? own.mass : own.count;
      if (x < target && target - x <= y) sm.bin = 255 - t, sm.above = before, sm.at = own;
    }
    if (n > 1) cl.sync();                              // (nobody clears what another still reads)
    else __syncthreads();
    p.key += sm.bin << shift;
    p.above = sm.above;
    p.at = sm.at;
    bits = shift;
    __syncthreads();
  } while (bits > 0);
  return p;
}

template <class T>
__device__ __forceinline__ float logit_at(const T* row, int i);
template <>
__device__ __forceinline__ float logit_at(const float* row, int i) { return __ldg(row + i); }
template <>
__device__ __forceinline__ float logit_at(const uint16_t* row, int i) { return bf16_bits_to_f32(__ldg(row + i)); }

// f(on, id, logit) for the elements [lo, hi) of a row, lo a multiple of 8, warp by warp.
template <class T, class F>
__device__ __forceinline__ void each_logit(const T* row, int lo, int hi, F f) {
  for (int i = lo + (threadIdx.x & ~31) * 8; i < hi; i += kThreads * 8) {
    const int c = i + (threadIdx.x & 31) * 8;
    float v[8];
    if (c + 8 <= hi) {
      Vec8<T>::load(row + c, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = c + e < hi ? logit_at(row, c + e) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) f(c + e < hi, c + e, v[e]);
  }
}

template <class T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleArgs a) {
  __shared__ Shared shared;
  Shared& sm = shared;
  cg::cluster_group cl = cg::this_cluster();
  const int n = a.cluster, rank = n > 1 ? (int)cl.block_rank() : 0, t = threadIdx.x;
  const long long r = blockIdx.x / n;
  const int V = a.vocab, per = ((V + n - 1) / n + 7) / 8 * 8, lo = min(V, rank * per), hi = min(V, lo + per);
  const T* row = static_cast<const T*>(a.logits) + r * a.stride;
  auto meet = [&] {
    if (n > 1) cl.sync();
    else __syncthreads();
  };
  if (n > 1) cl.barrier_arrive();
  tc::pdl_wait();
  tc::pdl_trigger();
  const float temp = a.temperature ? __ldg(a.temperature + r) : 1.f, top_p = a.top_p ? __ldg(a.top_p + r) : 1.f,
              min_p = a.min_p ? __ldg(a.min_p + r) : 0.f;
  const int top_k = a.top_k ? __ldg(a.top_k + r) : 0;
  const double u = __ldg(a.u + r);

  // ---- the largest logit
  Told mine;
  {
    float top = -INFINITY;
    bool bad = false;
    each_logit(row, lo, hi, [&](bool on, int, float x) {
      if (!on) return;
      top = fmaxf(top, x);
      bad |= !(x <= 3.40282347e38f);                   // NaN or +inf
    });
#pragma unroll
    for (int w = 16; w; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
    if ((t & 31) == 0) sm.fred[t >> 5] = top;
    if (t == 0) sm.n_list = 0u;
    mine.bad = __syncthreads_or(bad);
    for (int i = 0; i < kThreads / 32; ++i) top = fmaxf(top, sm.fred[i]);
    mine.top = top;
  }
  auto tell = [&](int what) {
    if (t < n) *(n > 1 ? cl.map_shared_rank(&sm.told[what][rank], t) : &sm.told[what][0]) = mine;
    meet();
  };
  mine.all = mine.near = {0ull, 0u};
  if (n > 1) cl.barrier_wait();                        // (the others have started)
  tell(0);
  float top = -INFINITY;
  bool bad = !(temp >= 0.f && temp <= 3.40282347e38f) || isnan(top_p) || isnan(min_p) || !(u >= 0. && u < 1.);
  for (int z = 0; z < n; ++z) top = fmaxf(top, sm.told[0][z].top), bad |= sm.told[0][z].bad != 0;
  bad |= top == -INFINITY;
  auto give = [&](int id, float prob, int kept) {
    if (rank == 0 && t == 0) {
      a.ids[r] = id;
      if (a.probs) a.probs[r] = prob;
      if (a.kept) a.kept[r] = kept;
    }
  };
  if (bad) {                                           // (every CTA of the cluster alike, here and below)
    if (rank == 0 && t == 0) atomicCAS(a.err, 0, (int)MCD_ERR_INVALID_ARG);
    give(-1, 0.f, 0);
    return;
  }
  const float z_top = __fdiv_rn(top, temp);
  const bool has_k = top_k > 0 && top_k < V, has_p = top_p < 1.f;
  const bool greedy = temp == 0.f || !(fabsf(z_top) <= 3.40282347e38f) || top_k == 1 || top_p <= 0.f;
  const float near = greedy ? top : top - kNear * temp;
  const uint32_t w_min = min_p > 0.f ? max(1u, (uint32_t)ceil((double)fminf(min_p, 1.f) * 2147483648.)) : 1u;
  auto weight = [&](float x) {
    if (greedy) return x >= top ? 1u : 0u;
    return __float2uint_rd(__fmul_rn(exp32_cw(__fsub_rn(__fdiv_rn(x, temp), z_top)), 2147483648.f));
  };
  auto from_row = [&](auto key, auto want) {
    return [=](auto f) {
      each_logit(row, lo, hi, [&](bool on, int id, float x) {
        const uint32_t k = key_of(x), w = on ? weight(x) : 0u;
        f(on && w > 0u && want(k, (uint32_t)id, w), key(k, (uint32_t)id), w);
      });
    };
  };
  auto from_list = [&](auto key, auto want) {
    return [=, &sm](auto f) {
      const int count = (int)sm.n_list;
      for (int i = t & ~31; i < count; i += kThreads) {
        const int j = i + (t & 31);
        const bool on = j < count;
        const uint32_t k = on ? sm.key[j] : 0u, id = on ? sm.id[j] : 0u, w = on ? sm.w[j] : 0u;
        f(on && want(k, id, w), key(k, id), w);
      }
    };
  };

  // ---- ids near the maximum to the first CTA's list; the sum of all weights where a cut or the draw needs it
  const bool whole = !has_k && !greedy;
  {
    Tally all{0ull, 0u}, close{0ull, 0u};
    Shared& home = *(n > 1 ? cl.map_shared_rank(&sm, 0) : &sm);
    each_logit(row, lo, hi, [&](bool on, int id, float x) {
      uint32_t w = 0u;
      if (on && (whole || x >= near)) w = weight(x);
      all.mass += w;
      const bool listed = on && x >= near && w > 0u;
      const unsigned mask = __ballot_sync(0xffffffffu, listed);
      if (!mask) return;
      uint32_t at = 0u;
      if ((t & 31) == __ffs(mask) - 1) at = atomicAdd(&home.n_list, (uint32_t)__popc(mask));
      at = __shfl_sync(0xffffffffu, at, __ffs(mask) - 1) + __popc(mask & ((1u << (t & 31)) - 1u));
      if (listed) {
        close.mass += w;
        ++close.count;
        if (at < (uint32_t)kList) home.key[at] = key_of(x), home.id[at] = (uint32_t)id, home.w[at] = w;
      }
    });
    mine.all = block_sum(sm, all);
    mine.near = block_sum(sm, close);
  }
  tell(1);
  Tally all{0ull, 0u}, close{0ull, 0u};
  for (int z = 0; z < n; ++z) {
    all.mass += sm.told[1][z].all.mass;
    close.mass += sm.told[1][z].near.mass, close.count += sm.told[1][z].near.count;
  }
  const bool listed = close.count <= (uint32_t)kList &&
                      (greedy || (has_k ? close.count >= (uint32_t)top_k
                                        : has_p && (double)close.mass >= ceil((double)top_p * (double)all.mass)));
  const int id_bits = 32 - __clz(V);                   // (V - 1 - id < 2^id_bits)
  auto by_key = [](uint32_t k, uint32_t) { return k; };
  auto by_id = [V](uint32_t, uint32_t id) { return (uint32_t)(V - 1) - id; };

  // The cuts and the draw, from the list (m = 1: the first CTA alone) or from the row (m = n).
  auto finish = [&](int m, auto from) {
    // counts and weights of what `want` takes, of all CTAs that take part
    auto tally = [&](auto want) {
      Tally x{0ull, 0u};
      from(by_key, want)([&](bool on, uint32_t, uint32_t w) {
        if (on) x.mass += w, ++x.count;
      });
      x = block_sum(sm, x);
      if (m > 1) {
        mine.all = x;
        tell(2);
        x = {0ull, 0u};
        for (int z = 0; z < m; ++z) x.mass += sm.told[2][z].all.mass, x.count += sm.told[2][z].all.count;
        meet();
      }
      return x;
    };
    auto any = [](uint32_t, uint32_t, uint32_t) { return true; };
    uint32_t cut = 0u, last = 0xffffffffu;             // larger keys are left, and of this one the ids up to `last`
    unsigned long long mass = all.mass;
    const uint32_t key_top = key_of(top);
    bool ties = false;
    uint32_t n_ties = 0u;
    if (greedy) {
      cut = key_top, n_ties = 1u, ties = true;
    } else {
      if (has_k) {
        // (ids without weight are behind all others)
        const Tally some = listed ? close : tally(any);
        mass = some.mass;
        if ((uint32_t)top_k < some.count) {
          const Pick p = pick(sm, m, 0u, 32, false, (unsigned long long)top_k, from(by_key, any));
          cut = p.key;
          n_ties = (uint32_t)top_k - p.above.count;
          ties = n_ties < p.at.count;
          mass = p.above.mass + p.at.mass / p.at.count * n_ties;
        }
      }
      if (has_p) {
        // (with top_p < 1 and mass < 2^50, the product is at most mass)
        const unsigned long long need = max(1ull, (unsigned long long)ceil((double)top_p * (double)mass));
        const uint32_t c = cut;
        const Pick p = pick(sm, m, 0u, 32, true, min(need, mass), from(by_key, [c](uint32_t k, uint32_t, uint32_t) { return k >= c; }));
        const unsigned long long one = p.at.mass / p.at.count;
        cut = p.key;
        n_ties = (uint32_t)((min(need, mass) - p.above.mass + one - 1) / one);
        ties = n_ties < p.at.count;
      }
    }
    if (ties) {
      const uint32_t c = cut;
      const Pick p = pick(sm, m, 0u, id_bits, false, n_ties, from(by_id, [c](uint32_t k, uint32_t, uint32_t) { return k == c; }));
      last = (uint32_t)(V - 1) - p.key;
    }
    auto left = [=](uint32_t k, uint32_t id, uint32_t w) { return (k > cut || (k == cut && id <= last)) && w >= (greedy ? 0u : w_min); };
    const Tally x = tally(left);
    const unsigned long long drawn = min((unsigned long long)floor(u * (double)x.mass), x.mass - 1);
    const Pick p = pick(sm, m, 0u, id_bits, true, drawn + 1, from(by_id, left));
    give(V - 1 - (int)p.key, (float)((double)p.at.mass / (double)x.mass), (int)x.count);
  };
  if (listed) {
    if (rank == 0) finish(1, from_list);
  } else {
    finish(n, from_row);
  }
}

// CTAs of a row: enough that each has kSlice ids at most.
constexpr int kSlice = 8192;
int cluster_for(int vocab) {
  int n = 1;
  while (n < kMaxCluster && vocab > n * kSlice) n *= 2;
  return n;
}

template <class T>
cudaError_t launch_sample(SampleArgs a, int n_rows, cudaStream_t st) {
  a.cluster = cluster_for(a.vocab);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n_rows * a.cluster);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = a.cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T>, a);
}

}  // namespace
}  // namespace rows
}  // namespace mcd

using namespace mcd;

extern "C" mcd_status mcd_sample_rows(int32_t n_rows, int32_t vocab, const void* logits, int64_t stride, int32_t dtype,
                                      const float* temperature, const int32_t* top_k, const float* top_p,
                                      const float* min_p, const double* u, int32_t* ids, float* probs, int32_t* kept,
                                      int32_t* err, void* stream) {
  using namespace rows;
  if (n_rows < 0 || vocab <= 0 || !err) return MCD_ERR_INVALID_ARG;
  if (dtype != MCD_WEIGHT_F32 && dtype != MCD_WEIGHT_BF16) return MCD_ERR_UNSUPPORTED;
  if (vocab > kMaxVocabRows || n_rows > (1 << 27)) return MCD_ERR_UNSUPPORTED;
  if (n_rows == 0) return MCD_OK;
  if (!logits || !u || !ids || stride < vocab) return MCD_ERR_INVALID_ARG;
  const Block in{logits, stride, n_rows, vocab, bytes_of(dtype)};
  if (!in.aligned()) return MCD_ERR_UNSUPPORTED;
  const SampleArgs a{logits, stride, vocab, 1, temperature, top_k, top_p, min_p, u, ids, probs, kept, err};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return cuda_status(dtype == MCD_WEIGHT_F32 ? launch_sample<float>(a, n_rows, st) : launch_sample<uint16_t>(a, n_rows, st));
}
