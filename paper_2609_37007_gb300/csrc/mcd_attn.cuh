// Shared by the kernels of mcd_paged_attention.
//
// The mathematics, per query vector q of a row (keys j over the visible positions):
//   s_j = scale q . k_j,  m = max s_j,  l = sum e^(s_j - m),  o = sum e^(s_j - m) v_j / l
// in one pass over the keys with a running m, l and unnormalised o (rescaled by e^(m_old - m_new) when
// m grows); in base 2: e^(s - m) = 2^(c q.k - max c q.k), c = scale log2(e).  Parts of the keys are
// joined by the same rule.
//
// The query vectors of one KV head (its group of query heads x the sequence's new rows, "packed"
// vector p = row * group + head of the group) read the same keys, so a CTA takes a tile of packed vectors
// of one (sequence, KV head).
#pragma once
#include <cooperative_groups.h>
#include <cuda.h>

#include "mcd_cache.cuh"

namespace mcd {
namespace paged {

struct AttnArgs {
  mcd_paged_kv kv;
  mcd_chunks ch;
  const void* q;
  void* out;
  const uint32_t* mask;
  int* err;
  long long q_stride, out_stride;
  int layer, group, mask_words;
  int splits;              // parts of a sequence's keys
  int least_vecs;          // the chunk kernel takes sequences with more packed vectors than this
  float* part;             // workspace of the parts (null: the CTAs of a cluster join them)
  float c;                 // scale * log2(e)
  int ranked;              // sequences are taken in the order of their tokens (by_tokens)
};

// CTAs start in the order of their numbers, and a long one that starts last is waited for alone: the sequences with most
// tokens come first.
constexpr int kRanked = 128;           // sequences that are put in order

// The sequence of rank `at`, ties in the order of their numbers.  The whole block calls it, of kRanked threads at least.
__device__ __forceinline__ int by_tokens(const mcd_chunks& ch, int at) {
  __shared__ __align__(16) int tokens[kRanked];
  __shared__ int found;
  const int i = threadIdx.x;
  int mine = -1;
  if (i < kRanked) {
    if (i < ch.n_seqs) {
      const Seq q = load_seq(ch, i);
      mine = q.n > 0 ? q.cached + q.n : 0;
    }
    tokens[i] = mine;
  }
  __syncthreads();
  if (i < ch.n_seqs) {
    int rank = 0;
    for (int n = 0; n < ch.n_seqs; n += 4) {           // (places behind the last sequence: -1)
      const int4 o = *reinterpret_cast<const int4*>(tokens + n);
      rank += (o.x > mine || (o.x == mine && n < i)) + (o.y > mine || (o.y == mine && n + 1 < i)) +
              (o.z > mine || (o.z == mine && n + 2 < i)) + (o.w > mine || (o.w == mine && n + 3 < i));
    }
    if (rank == at) found = i;
  }
  __syncthreads();
  return __reduce_max_sync(0xffffffffu, found);        // (a uniform register)
}

// Whether packed vectors of row i (of the sequence's new rows) see key `pos`; keys below q.cached are seen by all.
__device__ __forceinline__ bool sees(const AttnArgs& a, const Seq& q, int i, int pos) {
  const int j = pos - q.cached;
  if (j < 0) return true;
  if (j >= q.n || i >= q.n) return false;
  if (!a.mask) return j <= i;
  return (__ldg(a.mask + (long long)(q.row0 + i) * a.mask_words + (j >> 5)) >> (j & 31)) & 1u;
}

// What row i's unnormalised o is multiplied with, l the sum of its weights.  A sum of zero: the row sees nothing and is
// zeros, or every key that it sees scores -inf (each has weight 0, as beside a finite score) and 0 / 0 is NaN.
__device__ __forceinline__ float without_weights(const uint32_t* mask_row, int n) {
  uint32_t any = 0;
  for (int j = 0; j < n; j += 32) any |= __ldg(mask_row + (j >> 5)) & (n - j >= 32 ? 0xffffffffu : (1u << (n - j)) - 1u);
  return any ? NAN : 0.f;
}
// (behind a call: in line it takes the chunk and step kernels' last registers, 1 % of their time)
static __device__ __noinline__ float without_weights_call(const uint32_t* mask_row, int n) { return without_weights(mask_row, n); }
template <bool kCall = true>
__device__ __forceinline__ float normaliser(const AttnArgs& a, const Seq& q, int i, float l) {
  if (l != 0.f) return 1.f / l;
  if (!a.mask || q.cached > 0) return NAN;             // (without a mask it sees itself)
  const uint32_t* row = a.mask + (long long)(q.row0 + i) * a.mask_words;
  return kCall ? without_weights_call(row, q.n) : without_weights(row, q.n);
}

// Place (elements) of position pos of KV head h in the layer's pages; -1 for a page outside the pool.
__device__ __forceinline__ long long key_at(const AttnArgs& a, int s, int h, int pos) {
  const int page = __ldg(a.ch.table + (long long)s * a.ch.table_stride + pos / a.kv.page_size);
  if (page < 0 || page >= a.kv.n_pages) {
    report(a.err, MCD_ERR_INVALID_ARG);
    return -1;
  }
  return a.layer * a.kv.layer_stride + page * a.kv.page_stride + h * a.kv.head_stride +
         pos % a.kv.page_size * a.kv.token_stride;
}

// 2^x by the hardware's approximation (relative error 2^-22).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <class T>
__device__ __forceinline__ float4 load4(const T* p);
template <>
__device__ __forceinline__ float4 load4<float>(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
template <>
__device__ __forceinline__ float4 load4<uint16_t>(const uint16_t* p) {
  const uint2 w = __ldg(reinterpret_cast<const uint2*>(p));
  return make_float4(bf16_lo_f32(w.x), bf16_hi_f32(w.x), bf16_lo_f32(w.y), bf16_hi_f32(w.y));
}
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(uint16_t* p, float4 v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}

// Packed vectors p0 + r of a tile (r < 4096): row of the sequence and head of the group without a division each:
// floor(t / group) = t ceil(2^16 / group) >> 16 for t < 2^16 / group.
struct Pack {
  int row0, head0, inverse, group;
  __device__ __forceinline__ Pack(int p0, int group) : row0(p0 / group), head0(p0 - row0 * group), inverse((65535 + group) / group), group(group) {}
  __device__ __forceinline__ int row(int r) const { return row0 + ((head0 + r) * inverse >> 16); }
  __device__ __forceinline__ int head(int r) const { return head0 + r - ((head0 + r) * inverse >> 16) * group; }
};
// Elements of vector r in rows of `stride` elements.
template <int D>
__device__ __forceinline__ long long vec_at(const Pack& v, const Seq& q, int h, int r, long long stride) {
  return (q.row0 + v.row(r)) * stride + (h * v.group + v.head(r)) * D;
}

// Part z of the keys [0, n_keys), in whole tiles of `tile` keys.
struct Span {
  int lo, hi;
};
__device__ __forceinline__ Span part_of(int n_keys, int z, int splits, int tile) {
  const int per = ((n_keys + splits - 1) / splits + tile - 1) / tile * tile;
  const long long lo = min((long long)z * per, (long long)n_keys);
  return {(int)lo, (int)min((long long)n_keys, lo + per)};
}

// A warp's bounded wait (the same answer in every lane).  The test alone where the phase is over: a look at the abort
// flag beside it doubled the 64 cycles that it takes, six times a pair of tiles in the warp that issues.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, int* err, volatile int* abort_flag) {
  constexpr unsigned long long kWait = 2000000000ull;
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  const uint64_t t0 = globaltimer();
  for (int n = 1;; ++n) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if (n % 16) continue;
    const bool given_up = *abort_flag != 0, late = globaltimer() - t0 > kWait;
    if (__any_sync(0xffffffffu, given_up || late)) {
      if ((threadIdx.x & 31) == 0) {
        if (!given_up) report(err, MCD_ERR_TIMEOUT);
        *abort_flag = 1;
      }
      return false;
    }
  }
}

// Box of a page: places t0 .. of KV head h, dimensions d .. d + 63, in 128-byte swizzled rows.
__device__ __forceinline__ void tma_page(void* dst, const CUtensorMap* map, int d, int t0, int h, int page, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
          smem_u32(dst)),
      "l"(map), "r"(d), "r"(t0), "r"(h), "r"(page), "r"(smem_u32(bar))
      : "memory");
}

// Joins the parts of `vecs` packed vectors that the CTAs of a cluster hold in the same places of their shared
// memory: o [vec][pitch] unnormalised, m and l [vec].  Each CTA takes its share of the outputs.  A part without keys has
// m = -inf and l = 0.
template <class T, int D>
__device__ __forceinline__ void join_cluster(const AttnArgs& a, const Seq& q, int h, const Pack& pack, int vecs, float* o, int pitch,
                                             float* m, float* l) {
  namespace cg = cooperative_groups;
  cg::cluster_group cl = cg::this_cluster();
  cl.sync();
  const int n = (int)cl.num_blocks(), threads = (int)blockDim.x;
  for (int t = (int)cl.block_rank() * threads + threadIdx.x; t < vecs * (D / 4); t += n * threads) {
    const int r = t / (D / 4), d = t % (D / 4) * 4;
    float mx = -INFINITY;
    for (int z = 0; z < n; ++z) mx = fmaxf(mx, *cl.map_shared_rank(m + r, z));
    const float base = mx == -INFINITY ? 0.f : mx;
    float sum = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int z = 0; z < n; ++z) {
      const float w = exp2f(*cl.map_shared_rank(m + r, z) - base);
      const float4 y = *reinterpret_cast<const float4*>(cl.map_shared_rank(o + r * pitch + d, z));
      sum = fmaf(w, *cl.map_shared_rank(l + r, z), sum);
      x.x = fmaf(w, y.x, x.x), x.y = fmaf(w, y.y, x.y), x.z = fmaf(w, y.z, x.z), x.w = fmaf(w, y.w, x.w);
    }
    const float f = normaliser(a, q, pack.row(r), sum);
    store4(static_cast<T*>(a.out) + vec_at<D>(pack, q, h, r, a.out_stride) + d, make_float4(x.x * f, x.y * f, x.z * f, x.w * f));
  }
  cl.sync();                                           // nobody leaves while others read
}

__device__ __forceinline__ bool bf16x2_finite(uint32_t w) {
  return (w & 0x7F80u) != 0x7F80u && (w & 0x7F800000u) != 0x7F800000u;
}

// Launch with clusters of `cluster` CTAs along x.
template <class K, class... Args>
cudaError_t launch_clusters(K* kernel, dim3 grid, int threads, int cluster, size_t smem, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// The shared-memory opt-in is a property of the function: set once per device.
template <class K>
cudaError_t opt_in(K* kernel, int bytes, std::atomic<unsigned>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned bit = 1u << (dev & 31);
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_acq_rel);
  return e;
}

// Tensor map of one layer's pages for tma_page, boxes of `rows` places (false: no driver).
bool page_map(CUtensorMap* map, const mcd_paged_kv& kv, const void* pool, int layer, int rows);

// Sequences with more than a.least_vecs packed vectors, bf16 (mcd_attn_chunk.cu).
cudaError_t launch_chunk(const AttnArgs& a, cudaStream_t st);

}  // namespace paged
}  // namespace mcd
