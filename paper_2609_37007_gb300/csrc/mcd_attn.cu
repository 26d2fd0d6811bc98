// mcd_paged_attention (include/mcd_cache.h).
//
// The mathematics, per query vector q of a row (keys j over the visible positions):
//   s_j = scale q . k_j,  m = max s_j,  l = sum e^(s_j - m),  o = sum e^(s_j - m) v_j / l
// in one pass over the keys with a running m, l and unnormalised o (rescaled by e^(m_old - m_new) when
// m grows); in base 2: e^(s - m) = 2^(c q.k - c max q.k), c = scale log2(e).  Parts of the keys are
// joined by the same rule.
//
// The query vectors of one KV head (its group of query heads x the sequence's new rows, "packed"
// vector p = row * group + head of the group) read the same keys, so a CTA takes a tile of packed vectors
// of one (sequence, KV head).
#include <algorithm>

#include "mcd_cache.cuh"

namespace mcd {
namespace paged {
namespace {

struct AttnArgs {
  mcd_paged_kv kv;
  mcd_chunks ch;
  const void* q;
  void* out;
  const uint32_t* mask;
  int* err;
  long long q_stride, out_stride;
  int layer, group, mask_words;
  float c;                 // scale * log2(e)
};

// Whether packed vectors of row i (of the sequence's new rows) see key `pos`; keys below q.cached are seen by all.
__device__ __forceinline__ bool sees(const AttnArgs& a, const Seq& q, int i, int pos) {
  const int j = pos - q.cached;
  if (j < 0) return true;
  if (j >= q.n || i >= q.n) return false;
  if (!a.mask) return j <= i;
  return (__ldg(a.mask + (long long)(q.row0 + i) * a.mask_words + (j >> 5)) >> (j & 31)) & 1u;
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

// ---- plain fp32 arithmetic -------------------------------------------------------------------------
// A CTA of 16 x 16 threads takes 16 RM packed vectors against tiles of 64 keys: thread (ty, tx) has rows
// ty RM .. and keys tx + 16 c of the scores, then dimensions 4 tx .. (+ 64) of the same rows of o.
// The probabilities pass between the 16 threads of a row through shared memory.
constexpr int kFN = 64;
constexpr int kFThreads = 256;

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

template <int D, int RM>
struct FSmem {
  float q[16 * RM][D + 4], k[kFN][D + 4], v[kFN][D], p[16 * RM][kFN + 4];
};

template <class T, int D, int RM>
__global__ void __launch_bounds__(kFThreads) attn_f32_kernel(const AttnArgs a) {
  extern __shared__ __align__(16) uint8_t f_smem[];
  FSmem<D, RM>& sm = *reinterpret_cast<FSmem<D, RM>*>(f_smem);
  constexpr int kBM = 16 * RM, kDC = D / 64;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int h = blockIdx.y, s = blockIdx.z;
  tc::pdl_wait();
  tc::pdl_trigger();
  const Seq q = load_seq(a.ch, s);
  if (q.n < 0 && blockIdx.x == 0 && h == 0 && threadIdx.x == 0) report(a.err, MCD_ERR_INVALID_ARG);
  const long long vecs = (long long)max(q.n, 0) * a.group, p0 = (long long)blockIdx.x * kBM;
  if (p0 >= vecs) return;
  const int last_row = (int)min((long long)q.n - 1, (p0 + kBM - 1) / a.group);
  const int n_keys = a.mask ? q.cached + q.n : q.cached + last_row + 1;

  for (int i = threadIdx.x; i < kBM * (D / 4); i += kFThreads) {
    const int r = i / (D / 4), d = i % (D / 4) * 4;
    const long long p = p0 + r;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (p < vecs)
      x = load4(static_cast<const T*>(a.q) + (q.row0 + p / a.group) * a.q_stride + (h * a.group + p % a.group) * D + d);
    *reinterpret_cast<float4*>(&sm.q[r][d]) = x;
  }
  float m[RM], l[RM];
  float4 o[RM][kDC];
#pragma unroll
  for (int r = 0; r < RM; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < kDC; ++c) o[r][c] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  for (int k0 = 0; k0 < n_keys; k0 += kFN) {
    __syncthreads();
    for (int i = threadIdx.x; i < kFN * (D / 4); i += kFThreads) {
      const int r = i / (D / 4), d = i % (D / 4) * 4;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
      if (k0 + r < n_keys) {
        const long long at = key_at(a, s, h, k0 + r);
        if (at >= 0) {
          x = load4(static_cast<const T*>(a.kv.k) + at + d);
          y = load4(static_cast<const T*>(a.kv.v) + at + d);
        }
      }
      *reinterpret_cast<float4*>(&sm.k[r][d]) = x;
      *reinterpret_cast<float4*>(&sm.v[r][d]) = y;
    }
    __syncthreads();
    float z[RM][4];
#pragma unroll
    for (int r = 0; r < RM; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c) z[r][c] = 0.f;
#pragma unroll 4
    for (int d = 0; d < D; d += 4) {
      float4 kk[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) kk[c] = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * c][d]);
#pragma unroll
      for (int r = 0; r < RM; ++r) {
        const float4 qq = *reinterpret_cast<const float4*>(&sm.q[ty * RM + r][d]);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          z[r][c] = fmaf(qq.x, kk[c].x, fmaf(qq.y, kk[c].y, fmaf(qq.z, kk[c].z, fmaf(qq.w, kk[c].w, z[r][c]))));
      }
    }
    const bool edge = k0 + kFN > q.cached;             // some key of the tile may be hidden from some row
#pragma unroll
    for (int r = 0; r < RM; ++r) {
      const int row = (int)((p0 + ty * RM + r) / a.group);
      bool see[4];
      float mx = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        see[c] = !edge || sees(a, q, row, k0 + tx + 16 * c);
        z[r][c] = see[c] ? z[r][c] * a.c : -INFINITY;
        mx = fmaxf(mx, z[r][c]);
      }
#pragma unroll
      for (int w = 8; w; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float mn = fmaxf(m[r], mx), base = mn == -INFINITY ? 0.f : mn, f = exp2f(m[r] - base);
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float p = exp2f(z[r][c] - base);
        sum += see[c] ? p : 0.f;
        sm.p[ty * RM + r][tx + 16 * c] = see[c] ? p : -0.f;      // (hidden: the sign says so)
      }
      m[r] = mn;
      l[r] = l[r] * f + sum;                           // this thread's share of the row
#pragma unroll
      for (int c = 0; c < kDC; ++c) o[r][c].x *= f, o[r][c].y *= f, o[r][c].z *= f, o[r][c].w *= f;
    }
    __syncwarp();
    const int nk = min(kFN, n_keys - k0);
    for (int j = 0; j < nk; ++j) {
      float4 vv[kDC];
#pragma unroll
      for (int c = 0; c < kDC; ++c) vv[c] = *reinterpret_cast<const float4*>(&sm.v[j][tx * 4 + 64 * c]);
#pragma unroll
      for (int r = 0; r < RM; ++r) {
        const float p = sm.p[ty * RM + r][j];
        if (edge && __float_as_int(p) < 0) continue;   // hidden: v may be anything
#pragma unroll
        for (int c = 0; c < kDC; ++c) {
          o[r][c].x = fmaf(p, vv[c].x, o[r][c].x);
          o[r][c].y = fmaf(p, vv[c].y, o[r][c].y);
          o[r][c].z = fmaf(p, vv[c].z, o[r][c].z);
          o[r][c].w = fmaf(p, vv[c].w, o[r][c].w);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RM; ++r) {
    float sum = l[r];
#pragma unroll
    for (int w = 8; w; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
    const long long p = p0 + ty * RM + r;
    if (p >= vecs) continue;
    const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int c = 0; c < kDC; ++c)
      store4(static_cast<T*>(a.out) + (q.row0 + p / a.group) * a.out_stride + (h * a.group + p % a.group) * D + tx * 4 + 64 * c,
             make_float4(o[r][c].x * f, o[r][c].y * f, o[r][c].z * f, o[r][c].w * f));
  }
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

template <class T, int D, int RM>
cudaError_t launch_f32(const AttnArgs& a, cudaStream_t st) {
  static std::atomic<unsigned> done{0};
  const int bytes = (int)sizeof(FSmem<D, RM>);
  cudaError_t e = opt_in(attn_f32_kernel<T, D, RM>, bytes, done);
  if (e != cudaSuccess) return e;
  const long long tiles = ((long long)a.ch.max_rows * a.group + 16 * RM - 1) / (16 * RM);
  return tc::launch(true, attn_f32_kernel<T, D, RM>, dim3((unsigned)tiles, a.kv.n_kv_heads, a.ch.n_seqs), dim3(kFThreads), bytes,
                    st, a);
}
template <class T, int D>
cudaError_t launch_f32(const AttnArgs& a, cudaStream_t st) {
  return (long long)a.ch.max_rows * a.group <= 16 ? launch_f32<T, D, 1>(a, st) : launch_f32<T, D, 4>(a, st);
}

}  // namespace
}  // namespace paged
}  // namespace mcd

using namespace mcd;

extern "C" int64_t mcd_paged_attention_workspace(const mcd_paged_kv* kv, const mcd_chunks* chunks, int32_t n_q_heads) {
  (void)kv, (void)chunks, (void)n_q_heads;
  return 0;
}

extern "C" mcd_status mcd_paged_attention(const mcd_paged_kv* kv, int32_t layer, const mcd_chunks* chunks,
                                          int32_t n_q_heads, const void* q, int64_t q_stride, void* out,
                                          int64_t out_stride, float scale, const uint32_t* mask, int32_t mask_words,
                                          void* workspace, int64_t workspace_bytes, int32_t* err, void* stream) {
  using namespace paged;
  mcd_status s = check_kv(kv);
  if (s != MCD_OK) return s;
  if ((s = check_chunks(chunks, kv)) != MCD_OK) return s;
  if (layer < 0 || layer >= kv->n_layers || n_q_heads <= 0 || n_q_heads % kv->n_kv_heads || !err || !(scale > 0.f) ||
      !std::isfinite(scale))
    return MCD_ERR_INVALID_ARG;
  if (mask && (int64_t)mask_words * 32 < chunks->max_rows) return MCD_ERR_INVALID_ARG;
  if (n_q_heads / kv->n_kv_heads > 16) return MCD_ERR_UNSUPPORTED;
  if (no_rows(chunks)) return MCD_OK;
  if (!q || !out || q == out) return MCD_ERR_INVALID_ARG;
  const int64_t width = (int64_t)n_q_heads * kv->head_dim;
  if (q_stride < width || out_stride < width) return MCD_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || q_stride * esize(kv->dtype) % 16 || out_stride * esize(kv->dtype) % 16)
    return MCD_ERR_UNSUPPORTED;
  const int64_t need = mcd_paged_attention_workspace(kv, chunks, n_q_heads);
  if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return MCD_ERR_INVALID_ARG;
  const AttnArgs a{*kv, *chunks, q, out, mask, err, q_stride, out_stride, layer, n_q_heads / kv->n_kv_heads, mask_words,
                   scale * 1.4426950408889634f};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (kv->dtype == MCD_WEIGHT_F32)
    return cuda_status(kv->head_dim == 64 ? launch_f32<float, 64>(a, st) : launch_f32<float, 128>(a, st));
  return cuda_status(kv->head_dim == 64 ? launch_f32<uint16_t, 64>(a, st) : launch_f32<uint16_t, 128>(a, st));
}
