// mcd_rope_append and mcd_rope_freqs (include/mcd_cache.h): rows of a QKV product normalised,
// rotated and written to q and to the cache's pages.
//
// The mathematics: per head x -> x * gain / sqrt(mean x^2 + eps) (queries and keys, optional), then
// pair j turned by t = position * inv_freq[j]: (a, b) -> scale * (a cos t - b sin t, a sin t + b cos t).
// The angle is kept in turns as a 64-bit fixed-point fraction, F_j = frac(inv_freq[j] / 2 pi) * 2^64:
// position * F_j wraps at one turn by itself, so the reduction modulo one turn is exact at every
// position and costs one integer product.  The upper 32 bits of what is left go to sincospif as a float of
// half turns, whose 24 bits round them by up to 2^-26 turns (9e-8 radians), as any fp32 angle up to half a turn
// is.  A double product and its reduction would be bound by the GB300's few fp64 units.
//
// What bounds it: one read of the rows, one write of q and of the pages (HBM); for a few rows the
// chain row_start -> cached -> table -> store.  13,290 bf16 rows of 32 heads: 52.5 us, 4.1 TB/s (43 without norm and
// rotation; a copy of as many bytes takes 35); fp32 rows into an fp32 cache 80 us, 5.4 TB/s (a copy: 67).
#include <algorithm>

#include "mcd_cache.cuh"

namespace mcd {
namespace paged {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeRows = 4;           // rows that a CTA's threads hold at a time
constexpr int kRopeSteps = 4;          // of these, at most, one after another

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
  int layer, n_q, steps;
  float eps;
};

// Eight elements as they lie, and as fp32.
template <class T>
struct Raw8;
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __ldcs(reinterpret_cast<const float4*>(p));
    b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void get(uint64_t (&x)[4]) const {
    x[0] = pack2(a.x, a.y), x[1] = pack2(a.z, a.w), x[2] = pack2(b.x, b.y), x[3] = pack2(b.z, b.w);
  }
};
template <>
struct Raw8<uint16_t> {
  uint4 a;
  __device__ __forceinline__ void load(const uint16_t* p) { a = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void get(uint64_t (&x)[4]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = pack2(bf16_lo_f32(w[i]), bf16_hi_f32(w[i]));
  }
};
__device__ __forceinline__ void store8(float* p, const uint64_t (&x)[4]) {
  float4 u, v;
  unpack2(x[0], u.x, u.y), unpack2(x[1], u.z, u.w), unpack2(x[2], v.x, v.y), unpack2(x[3], v.z, v.w);
  reinterpret_cast<float4*>(p)[0] = u;
  reinterpret_cast<float4*>(p)[1] = v;
}
__device__ __forceinline__ void store8(uint16_t* p, const uint64_t (&x)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float u, v;
    unpack2(x[i], u, v);
    w[i] = pack_bf16x2(u, v);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void load_gain(uint64_t (&g)[4], const float* from) {
  const float4 u = __ldg(reinterpret_cast<const float4*>(from)), v = __ldg(reinterpret_cast<const float4*>(from) + 1);
  g[0] = pack2(u.x, u.y), g[1] = pack2(u.z, u.w), g[2] = pack2(v.x, v.y), g[3] = pack2(v.z, v.w);
}
// Neighbours (x.lo, x.hi), ..: pair e of x by angles (lo or hi of c[e / 2], s[e / 2]).
__device__ __forceinline__ void turn_neighbours(uint64_t (&x)[4], const uint64_t* c, const uint64_t* s) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float u, v, c0, c1, s0, s1;
    unpack2(x[e], u, v), unpack2(c[e / 2], c0, c1), unpack2(s[e / 2], s0, s1);
    const float cc = e % 2 ? c1 : c0, ss = e % 2 ? s1 : s0;
    x[e] = fma2(pack2(v, u), pack2(-ss, ss), mul2(x[e], pack2(cc, cc)));
  }
}

// Where a row goes: place of head 0 in the layer's pages (elements; -1: the row is nobody's or its
// sequence does not fit) and its position.
struct RowPlace {
  long long at;
  int pos;
};

// In: type of the qkv rows, Out: type of the cache.  A CTA takes a.steps times kRopeRows rows: a warp per row finds the
// rows' places, then every thread makes (row, pair) angles.  For the heads a thread keeps one row and two pieces of
// eight dimensions, both elements of eight pairs (D / 16 neighbouring lanes hold a head), so that its cosines, sines
// and gains stay in registers and no element crosses lanes; it goes through the heads in steps of its group,
// kAhead heads' loads in flight, the first ones before the row's place is known.
// (A piece and its pairs' other halves by shuffles: 110 instructions for 16 bytes, issue-bound, 60 us where this takes
// the time below.)
template <class In, class Out, int D>
__global__ void __launch_bounds__(kRopeThreads, 2) rope_append_kernel(const RopeArgs a) {
  constexpr int kLanes = D / 16, kGroup = kLanes * kRopeRows, kGroups = kRopeThreads / kGroup, kAhead = sizeof(In) == 2 ? 4 : 2;
  __shared__ unsigned long long turn[D / 2];           // F_j
  __shared__ float2 cs[kRopeRows * kRopeSteps][D / 2]; // (cos, sin) * scale
  __shared__ RowPlace place[kRopeRows * kRopeSteps];
  const int half = a.rope.rot_dim / 2, n_qk = a.n_q + a.kv.n_kv_heads, n_heads = n_qk + a.kv.n_kv_heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = threadIdx.x % kLanes, r = threadIdx.x / kLanes % kRopeRows, group = threadIdx.x / kGroup;
  // Lanes of the warp with the same head: a group.  With D = 64 a warp holds two, whose heads may be of different kinds, so
  // that only one of them takes the norm's sum.
  static_assert(kGroup == 16 || kGroup == 32, "a group is a warp or half of one");
  const unsigned same_head = kGroup == 32 ? 0xffffffffu : 0xffffu << (lane & 16);
  // first dimension of the two pieces; pairs are 8 t .. 8 t + 7 (behind the pairs: what is left, in order)
  const bool turned = t < half / 8;
  const int d0 = a.rope.interleaved || !turned ? 16 * t : 8 * t, d1 = a.rope.interleaved || !turned ? d0 + 8 : d0 + half;
  const int tile = blockIdx.x * (kRopeRows * a.steps);
  tc::pdl_wait();
  tc::pdl_trigger();
  const int n_rows = min(__ldg(a.ch.row_start + a.ch.n_seqs), a.ch.n_rows);
  const int rows = min(kRopeRows * a.steps, n_rows - tile);
  const In* src = static_cast<const In*>(a.qkv) + (tile + (long long)r) * a.qkv_stride;
  const int per_step = (n_heads + kAhead * kGroups - 1) / (kAhead * kGroups), n_it = per_step * a.steps;
  Raw8<In> raw[kAhead][2] = {};
  auto fetch = [&](int i, int step, int h0) {          // head i of the iteration that starts with (step, h0)
    const int head = h0 + i * kGroups;
    if (step * kRopeRows + r < rows && head < n_heads) {
      const In* p = src + step * (kRopeRows * a.qkv_stride) + head * D;
      raw[i][0].load(p + d0);
      raw[i][1].load(p + d1);
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(i, 0, group);
  if (threadIdx.x < half) {
    const double w = __ldg(a.rope.inv_freq + threadIdx.x) * 0.15915494309189535;   // turns per position
    turn[threadIdx.x] = (unsigned long long)((w - floor(w)) * 18446744073709551616.0);
  }
  for (int n = warp; n < rows; n += kRopeThreads / 32) {
    const int row = tile + n;
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
    if (lane == 0) place[n] = p;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * half; i += kRopeThreads) {
    const int row = i / half, j = i - row * half;
    const unsigned long long f = (unsigned long long)(long long)place[row].pos * turn[j];
    float sn, cn;
    sincospif((float)(int)(f >> 32) * 4.656612873077393e-10f, &sn, &cn);   // half turns in [-1, 1]
    cs[row][j] = make_float2(cn * a.rope.scale, sn * a.rope.scale);
  }
  __syncthreads();
  uint64_t cosv[4], sinv[4], gain[2][4];               // two of each an element
  const float* held = nullptr;                         // whose gains these are
  long long at = -1;
  Out* q_row = nullptr;
  int step = 0, h0 = group;
  for (int it = 0; it < n_it; ++it) {
    if (h0 == group) {                                 // new rows
      const int row = step * kRopeRows + r;
      if (step * kRopeRows >= rows) break;             // (the whole CTA)
      at = row < rows ? place[row].at : -1;
      q_row = static_cast<Out*>(a.q_out) + (tile + (long long)row) * a.q_stride;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool there = turned && row < rows;
        const float2 u = there ? cs[row][8 * t + 2 * e] : make_float2(1.f, 0.f);
        const float2 v = there ? cs[row][8 * t + 2 * e + 1] : make_float2(1.f, 0.f);
        cosv[e] = pack2(u.x, v.x);
        sinv[e] = pack2(u.y, v.y);
      }
    }
    const int h_now = h0;
    h0 += kAhead * kGroups;
    if (h0 >= per_step * kAhead * kGroups) h0 = group, ++step;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int head = h_now + i * kGroups;            // (the same in the lanes of same_head)
      uint64_t x[4], y[4];
      raw[i][0].get(x);
      raw[i][1].get(y);
      if (it + 1 < n_it) fetch(i, step, h0);           // (the next iteration's, on its way during this one)
      if (head >= n_heads) continue;
      if (head < n_qk) {
        const float* norm = head < a.n_q ? a.q_norm : a.k_norm;
        if (norm) {
          if (norm != held) {
            held = norm;
            load_gain(gain[0], norm + d0);
            load_gain(gain[1], norm + d1);
          }
          uint64_t squares = mul2(x[0], x[0]);
#pragma unroll
          for (int e = 1; e < 4; ++e) squares = fma2(x[e], x[e], squares);
#pragma unroll
          for (int e = 0; e < 4; ++e) squares = fma2(y[e], y[e], squares);
          float ss, odd;
          unpack2(squares, ss, odd);
          ss += odd;
#pragma unroll
          for (int m = kLanes / 2; m; m >>= 1) ss += __shfl_xor_sync(same_head, ss, m);
          const float f = rsqrtf(ss * (1.f / D) + a.eps);
          const uint64_t ff = pack2(f, f);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = mul2(x[e], mul2(ff, gain[0][e])), y[e] = mul2(y[e], mul2(ff, gain[1][e]));
        }
        if (turned) {
          if (a.rope.interleaved) {
            turn_neighbours(x, cosv, sinv);
            turn_neighbours(y, cosv + 2, sinv + 2);
          } else {
            const uint64_t minus = pack2(-1.f, -1.f);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint64_t u = x[e];
              x[e] = fma2(mul2(y[e], minus), sinv[e], mul2(u, cosv[e]));
              y[e] = fma2(u, sinv[e], mul2(y[e], cosv[e]));
            }
          }
        }
      }
      if (at < 0) continue;
      Out* to = head < a.n_q    ? q_row + head * D
                : head < n_qk   ? static_cast<Out*>(a.kv.k) + at + (head - a.n_q) * a.kv.head_stride
                                : static_cast<Out*>(a.kv.v) + at + (head - n_qk) * a.kv.head_stride;
      store8(to + d0, x);
      store8(to + d1, y);
    }
  }
  if (blockIdx.x == 0)
    for (int s = threadIdx.x; s < a.ch.n_seqs; s += kRopeThreads)
      if (load_seq(a.ch, s).n < 0) report(a.err, MCD_ERR_INVALID_ARG);
}

template <class In, class Out>
cudaError_t launch_rope(RopeArgs a, cudaStream_t st) {
  // as many steps as leave two CTAs (what an SM holds) for every SM
  a.steps = std::max(1, std::min(kRopeSteps, a.ch.n_rows / (2 * kRopeRows * sm_count())));
  const dim3 grid((unsigned)(((long long)a.ch.n_rows + kRopeRows * a.steps - 1) / (kRopeRows * a.steps)));
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
  const RopeArgs a{*kv, *chunks, *rope, qkv, q_out, positions, q_norm, k_norm, err, qkv_stride, q_stride, layer, n_q_heads, 1, eps};
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
