// mcd_rope_append and mcd_rope_freqs (include/mcd_cache.h): rows of a QKV product normalised,
// rotated and written to q and to the cache's pages.
//
// The mathematics: per head x -> x * gain / sqrt(mean x^2 + eps) (queries and keys, optional), then
// pair j turned by t = position * inv_freq[j]: (a, b) -> scale * (a cos t - b sin t, a sin t + b cos t).
// The angle is kept in turns as a 64-bit fixed-point fraction, F_j = frac(inv_freq[j] / 2 pi) * 2^64:
// position * F_j wraps at one turn by itself, so the reduction modulo 2 pi is exact at every
// position and costs one integer product; what is left of it (32 bits, 2^-33 turns) goes to
// sincospif.  A double product and its reduction would be bound by the GB300's few fp64 units.
//
// What bounds it: one read of the rows, one write of q and of the pages (HBM); for a few rows the
// chain row_start -> cached -> table -> store.
#include <algorithm>

#include "mcd_cache.cuh"

namespace mcd {
namespace paged {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeRows = 8;           // rows of a CTA's tile: one warp looks up each

struct RopeArgs {
  mcd_paged_kv kv;
  mcd_chunks ch;
  mcd_rope rope;
  const void* qkv;
  void* q_out;
  const int32_t* positions;
  const float *q_norm, *k_norm;
  int* err;
  long long qkv_stride, q_stride;
  int layer, n_q;
  float eps;
};

template <class T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&x)[8]) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
template <>
__device__ __forceinline__ void load8<uint16_t>(const uint16_t* p, float (&x)[8]) {
  const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo_f32(w[i]), x[2 * i + 1] = bf16_hi_f32(w[i]);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                                            pack_bf16x2(x[6], x[7]));
}

// Where a row goes: place of head 0 in the layer's pages (elements; -1: the row is nobody's or its
// sequence does not fit) and its position.
struct RowPlace {
  long long at;
  int pos;
};

// In: type of the qkv rows, Out: type of the cache.  A CTA takes tiles of kRopeRows rows: first a warp
// per row finds the row's place while the angles' factors are made, then all threads the (row, pair) angles,
// then eight elements of a head per thread (head_dim / 8 neighbouring lanes hold a head).
template <class In, class Out, int D>
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const RopeArgs a) {
  constexpr int kLanes = D / 8;                        // lanes of a head
  __shared__ unsigned long long turn[D / 2];           // F_j
  __shared__ float2 cs[kRopeRows][D / 2];              // (cos, sin) * scale of the tile's rows
  __shared__ RowPlace place[kRopeRows];
  const int half = a.rope.rot_dim / 2, n_heads = a.n_q + 2 * a.kv.n_kv_heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  tc::pdl_wait();
  tc::pdl_trigger();
  if (threadIdx.x < half) {
    const double w = __ldg(a.rope.inv_freq + threadIdx.x) * 0.15915494309189535;   // turns per position
    turn[threadIdx.x] = (unsigned long long)((w - floor(w)) * 18446744073709551616.0);
  }
  const int last = __ldg(a.ch.row_start + a.ch.n_seqs);
  const int n_rows = min(last, a.ch.n_rows);
  for (long long tile = (long long)blockIdx.x * kRopeRows; tile < n_rows; tile += (long long)gridDim.x * kRopeRows) {
    const int rows = (int)min((long long)kRopeRows, n_rows - tile);
    if (warp < rows) {
      const int row = (int)tile + warp;
      // (empty sequences share their start with the next one: the last of them has the row)
      const int s = warp_last_le(a.ch.n_seqs, [&](int i) { return (long long)__ldg(a.ch.row_start + i); }, row);
      const Seq q = load_seq(a.ch, s);
      RowPlace p{-1, 0};
      if (q.n > 0 && row >= q.row0 && row - q.row0 < q.n) {
        const int slot = q.cached + row - q.row0;
        const int page = __ldg(a.ch.table + (long long)s * a.ch.table_stride + slot / a.kv.page_size);
        if (page < 0 || page >= a.kv.n_pages) {
          if (lane == 0) report(a.err, MCD_ERR_INVALID_ARG);
        } else {
          p.at = a.layer * a.kv.layer_stride + page * a.kv.page_stride + slot % a.kv.page_size * a.kv.token_stride;
          p.pos = a.positions ? __ldg(a.positions + row) : slot;
        }
      }
      if (lane == 0) place[warp] = p;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * half; i += kRopeThreads) {
      const int r = i / half, j = i - r * half;
      const unsigned long long t = (unsigned long long)(long long)place[r].pos * turn[j];
      float sn, cn;
      sincospif((float)(int)(t >> 32) * 4.656612873077393e-10f, &sn, &cn);   // half turns in [-1, 1]
      cs[r][j] = make_float2(cn * a.rope.scale, sn * a.rope.scale);
    }
    __syncthreads();
    const int n_tasks = rows * n_heads * kLanes;
    for (int t0 = warp * 32; t0 < n_tasks; t0 += kRopeThreads) {
      const int t = t0 + lane;                         // (the lanes of a head are in or out together)
      const bool live = t < n_tasks;
      const int c = t % kLanes, rest = live ? t / kLanes : 0, r = rest / n_heads, head = rest - r * n_heads;
      const long long at = place[r].at, row = tile + r;
      float x[8];
      load8(static_cast<const In*>(a.qkv) + row * a.qkv_stride + (long long)head * D + c * 8, x);
      const bool is_v = head >= a.n_q + a.kv.n_kv_heads;
      const float* gain = head < a.n_q ? a.q_norm : a.k_norm;
      if (a.q_norm || a.k_norm) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
        for (int m = kLanes / 2; m; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
        if (gain && !is_v) {
          const float f = 1.f / sqrtf(ss * (1.f / D) + a.eps);
          float gv[8];
          load8(gain + c * 8, gv);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = x[e] * f * gv[e];
        }
      }
      if (half) {
        const int e0 = c * 8;
        if (a.rope.interleaved) {
          if (e0 < 2 * half && !is_v) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              const float2 w = cs[r][(e0 + e) / 2];
              const float u = x[e], v = x[e + 1];
              x[e] = u * w.x - v * w.y;
              x[e + 1] = u * w.y + v * w.x;
            }
          }
        } else {                                       // the partner's eight elements are half / 8 lanes away
          const bool low = e0 < half, in = e0 < 2 * half;
          const int from = in ? lane + (low ? half / 8 : -(half / 8)) : lane;
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = __shfl_sync(0xffffffffu, x[e], from);
          if (in && !is_v) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float2 w = cs[r][e0 + e - (low ? 0 : half)];
              x[e] = low ? x[e] * w.x - y[e] * w.y : y[e] * w.y + x[e] * w.x;
            }
          }
        }
      }
      if (!live || at < 0) continue;
      if (head < a.n_q) {
        store8(static_cast<Out*>(a.q_out) + row * a.q_stride + (long long)head * D + c * 8, x);
      } else {
        const int h = head - a.n_q - (is_v ? a.kv.n_kv_heads : 0);
        store8(static_cast<Out*>(is_v ? a.kv.v : a.kv.k) + at + h * a.kv.head_stride + c * 8, x);
      }
    }
    __syncthreads();                                   // the tile's tables are free again
  }
  if (blockIdx.x == 0)
    for (int s = threadIdx.x; s < a.ch.n_seqs; s += kRopeThreads)
      if (load_seq(a.ch, s).n < 0) report(a.err, MCD_ERR_INVALID_ARG);
}

template <class In, class Out>
cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st) {
  const int tiles = (a.ch.n_rows + kRopeRows - 1) / kRopeRows;
  const dim3 grid(std::min(tiles, sm_count() * 8));
  auto k = a.kv.head_dim == 64 ? rope_append_kernel<In, Out, 64> : rope_append_kernel<In, Out, 128>;
  return tc::launch(true, k, grid, dim3(kRopeThreads), 0, st, a);
}

}  // namespace
}  // namespace paged
}  // namespace mcd

using namespace mcd;

extern "C" mcd_status mcd_rope_append(const mcd_paged_kv* kv, int32_t layer, const mcd_chunks* chunks, int32_t n_q_heads,
                                      const void* qkv, int64_t qkv_stride, int32_t qkv_dtype, void* q_out,
                                      int64_t q_stride, const mcd_rope* rope, const int32_t* positions,
                                      const float* q_norm, const float* k_norm, float eps, int32_t* err, void* stream) {
  using namespace paged;
  mcd_status s = check_kv(kv);
  if (s != MCD_OK) return s;
  if ((s = check_chunks(chunks, kv)) != MCD_OK) return s;
  if (layer < 0 || layer >= kv->n_layers || n_q_heads <= 0 || !rope || !err || !(eps >= 0.f) || !std::isfinite(eps) ||
      !std::isfinite(rope->scale))
    return MCD_ERR_INVALID_ARG;
  if (rope->rot_dim < 0 || rope->rot_dim > kv->head_dim || (rope->rot_dim && !rope->inv_freq)) return MCD_ERR_INVALID_ARG;
  if (rope->rot_dim % 16 || n_q_heads > 4096) return MCD_ERR_UNSUPPORTED;
  if (qkv_dtype != MCD_WEIGHT_F32 && (qkv_dtype != MCD_WEIGHT_BF16 || kv->dtype != MCD_WEIGHT_BF16)) return MCD_ERR_UNSUPPORTED;
  if (no_rows(chunks)) return MCD_OK;
  if (!qkv || !q_out) return MCD_ERR_INVALID_ARG;
  const int64_t q_width = (int64_t)n_q_heads * kv->head_dim, width = q_width + 2ll * kv->n_kv_heads * kv->head_dim;
  if (qkv_stride < width || q_stride < q_width) return MCD_ERR_INVALID_ARG;
  if (!aligned16(qkv) || !aligned16(q_out) || qkv_stride * esize(qkv_dtype) % 16 || q_stride * esize(kv->dtype) % 16 ||
      !aligned16(q_norm) || !aligned16(k_norm))
    return MCD_ERR_UNSUPPORTED;
  const RopeArgs a{*kv, *chunks, *rope, qkv, q_out, positions, q_norm, k_norm, err, qkv_stride, q_stride, layer, n_q_heads, eps};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (kv->dtype == MCD_WEIGHT_F32) return cuda_status(launch_rope<float, float>(a, st));
  return cuda_status(qkv_dtype == MCD_WEIGHT_F32 ? launch_rope<float, uint16_t>(a, st) : launch_rope<uint16_t, uint16_t>(a, st));
}

extern "C" mcd_status mcd_rope_freqs(int32_t kind, int32_t rot_dim, double base, double factor, int32_t train_tokens,
                                     double beta_fast, double beta_slow, double* inv_freq, float* scale) {
  if (!inv_freq || rot_dim <= 0 || rot_dim % 2 || !(base > 1.0) || !std::isfinite(base) || !(factor >= 1.0) ||
      !std::isfinite(factor))
    return MCD_ERR_INVALID_ARG;
  const bool parts = kind == MCD_ROPE_BY_PARTS;
  if (kind < MCD_ROPE_PLAIN || kind > MCD_ROPE_BY_PARTS || (kind == MCD_ROPE_BASE && rot_dim == 2)) return MCD_ERR_INVALID_ARG;
  if (kind == MCD_ROPE_PLAIN && factor != 1.0) return MCD_ERR_INVALID_ARG;
  if (parts && (train_tokens < 1 || !(beta_slow > 0.0) || !(beta_fast > beta_slow) || !std::isfinite(beta_fast)))
    return MCD_ERR_INVALID_ARG;
  const double b = kind == MCD_ROPE_BASE ? base * std::pow(factor, rot_dim / (rot_dim - 2.0)) : base;
  // the pair whose frequency makes `turns` turns over the trained context, as a real number
  auto pair_of = [&](double turns) {
    return rot_dim * std::log(train_tokens / (turns * 6.283185307179586)) / (2.0 * std::log(base));
  };
  const double lo = parts ? pair_of(beta_fast) : 0.0, hi = parts ? pair_of(beta_slow) : 1.0;
  for (int j = 0; j < rot_dim / 2; ++j) {
    const double w = std::pow(b, -2.0 * j / rot_dim);
    double g = 0.0;                                    // share of the stretched frequency
    if (kind == MCD_ROPE_LINEAR) g = 1.0;
    if (parts) g = std::fmin(1.0, std::fmax(0.0, (j - lo) / (hi - lo)));
    inv_freq[j] = w * (1.0 - g) + w / factor * g;
  }
  if (scale) *scale = parts ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return MCD_OK;
}
