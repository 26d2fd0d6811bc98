// mcd_norm_rows (include/mcd_rows.h): residual sum, RMSNorm and rounding of rows, to 8 bits with a scale too.
//
// The mathematics, per row of n elements: r = x + residual; q = sum r^2, i = 1 / sqrt(q / n + eps), v = r i gain.  The scale of
// 8 bits is max |v| / 448 = i max |r gain| / 448, so that q and the maximum are found in one pass and joined once (a row whose
// r gain leaves fp32's range is looked at again); the row stays in registers between its load and its store.
// What bounds it: one read of x and the residual, one write of the sum and of y; for a few rows the chain load -> join -> store.
// 30,011 rows of 4,096, bf16 in, sum and residual, 8 bits out: 154 us, 5.6 TB/s (0.84 of a copy; bf16 out 161, fp32 sums and out
// 257 us or 6.7 TB/s).  A thread has 8 or 16 elements and a row as many threads as that takes, so that the SM's 2,048 threads have
// 64 bytes each on their way: 4,096 elements on 512 threads 156, on 256 of two chunks 157, on 128 of four 173 us; 1,024 on a warp
// of four chunks 89 against 72.  CTAs that stay and load the next row under the join took 296 (64 registers: half the threads).
#include <cmath>

#include "mcd_cache.cuh"
#include "mcd_rows.cuh"

namespace mcd {
namespace rows {
namespace {

struct NormArgs {
  const void *x, *res;
  void *sum, *y;
  const float* gain;
  float* scale;
  long long x_stride, res_stride, sum_stride, y_stride;
  int n_rows, width;
  int norm;
  float eps, inv_width;
};

using paged::add2;
using paged::fma2;
using paged::mul2;
using paged::pack2;
using paged::unpack2;

// Elements 8 c .. 8 c + 7 of a row in pairs, those from `width` on zeros.
template <class T>
__device__ __forceinline__ void load8(const void* base, long long row, long long stride, int c, int width, uint64_t (&v)[4]) {
  const T* p = static_cast<const T*>(base) + row * stride + 8 * c;
  float x[8];
  if (8 * c + 8 <= width) {
    Vec8<T>::load(p, x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 8 * c + e < width ? Vec8<T>::one(p[e]) : 0.f;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = pack2(x[2 * e], x[2 * e + 1]);
}
template <class T>
__device__ __forceinline__ void store8(void* base, long long row, long long stride, int c, int width, const uint64_t (&v)[4]) {
  T* p = static_cast<T*>(base) + row * stride + 8 * c;
  float x[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) unpack2(v[e], x[2 * e], x[2 * e + 1]);
  if (8 * c + 8 <= width) {
    Vec8<T>::store(p, x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (8 * c + e < width) p[e] = Vec8<T>::round(x[e]);
  }
}

// A team of kTeam threads takes a row, thread t its chunks t, t + kTeam, .. of 8 elements (kChunks at most).  Teams of a warp
// share a CTA of 128 threads.  Two CTAs of 1,024 an SM: 6,000 rows of 16,384 take 135 us (one: 187), fp32 sums and results 244 (272).
template <class TX, class TR, class TY, int kTeam, int kChunks>
__global__ void __launch_bounds__(kTeam < 128 ? 128 : kTeam, kTeam == 1024 ? 2 : 0) norm_kernel(const NormArgs a) {
  constexpr int kTeams = kTeam < 128 ? 128 / kTeam : 1;
  constexpr bool k8 = sizeof(TY) == 1;
  static_assert(kTeam == 32 || kTeam >= 128, "a team is a warp or a CTA");
  const int t = threadIdx.x % kTeam, n_chunks = (a.width + 7) / 8;
  const long long row = (long long)blockIdx.x * kTeams + threadIdx.x / kTeam;
  tc::pdl_wait();
  tc::pdl_trigger();
  if (row >= a.n_rows) return;                         // (a whole team)
  uint64_t v[kChunks][4];
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    const int c = t + i * kTeam;
    if (c < n_chunks) {
      load8<TX>(a.x, row, a.x_stride, c, a.width, v[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = 0ull;      // (two zeros)
    }
  }
  if (a.res) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int c = t + i * kTeam;
      if (c >= n_chunks) continue;
      uint64_t r[4];
      load8<TR>(a.res, row, a.res_stride, c, a.width, r);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = add2(v[i][e], r[e]);
    }
  }
  if (a.sum) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int c = t + i * kTeam;
      if (c < n_chunks) store8<TR>(a.sum, row, a.sum_stride, c, a.width, v[i]);
    }
  }
  uint64_t q2 = 0ull;
#pragma unroll
  for (int i = 0; i < kChunks; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) q2 = fma2(v[i][e], v[i][e], q2);
  // (one chunk's gains stay in registers; those of two would take a CTA's place on the SM, 12,000 rows of 8,192 169 us instead of 140, and
  // are read where they are wanted)
  uint64_t kept[4];
  auto load_gain = [&](int i, uint64_t (&g)[4]) {
    const int c = t + i * kTeam;
    if (a.gain && c < n_chunks) {
      load8<float>(a.gain, 0, 0, c, a.width, g);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = pack2(1.f, 1.f);
    }
  };
  auto gain_of = [&](int i, uint64_t (&g)[4]) {
    if (kChunks > 1) {
      load_gain(i, g);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = kept[e];
    }
  };
  if (kChunks == 1) load_gain(0, kept);
  // the largest |r gain|, of the thread's elements, or with `scaled` the largest |r f gain|
  auto largest = [&](bool scaled, float f) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      uint64_t g[4];
      gain_of(i, g);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x, y;
        unpack2(mul2(scaled ? mul2(v[i][e], pack2(f, f)) : v[i][e], g[e]), x, y);
        top = max3_nan(top, fabsf(x), fabsf(y));
      }
    }
    return top;
  };
  float q, top = 0.f;
  {
    float x, y;
    unpack2(q2, x, y);
    q = x + y;
    if (k8) top = largest(false, 1.f);
  }
  // (the order of the sum is fixed by the sizes)
  team_join<kTeam, k8>(q, top);
  // (a sum that is not finite: neither is the row, where 1 / inf would leave zeros)
  const float inv = !a.norm ? 1.f : q <= 3.40282347e38f ? rsqrtf(fmaf(q, a.inv_width, a.eps)) : NAN;
  float back = 1.f;
  if (k8) {
    if (a.norm && !(top >= 1e-30f && top <= 3.40282347e38f)) {      // r gain out of fp32's range, where v may be in it: once more, of v
      if (kTeam > 32) __syncthreads();                 // (the join before has been read)
      top = largest(true, inv);
      team_join<kTeam, k8>(q, top);                    // (q is not looked at again)
    } else {
      top *= inv;
    }
    const float s = max_nan(top * (1.f / 448.f), 1.17549435e-38f);
    back = __fdividef(1.f, s);                         // (s < 2^120: a maximum over 448)
    if (t == 0) a.scale[row] = s;
  }
  // (v in this order: r / rms is of the size of one, r gain may leave fp32's range)
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    const int c = t + i * kTeam;
    if (c >= n_chunks) continue;
    uint64_t g[4];
    gain_of(i, g);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[i][e] = mul2(mul2(v[i][e], pack2(inv, inv)), g[e]);
      if (k8) v[i][e] = mul2(v[i][e], pack2(back, back));
    }
    store8<TY>(a.y, row, a.y_stride, c, a.width, v[i]);
  }
}

template <class TX, class TR, class TY, int kTeam, int kChunks>
cudaError_t launch_norm(const NormArgs& a, cudaStream_t st) {
  constexpr int kTeams = kTeam < 128 ? 128 / kTeam : 1;
  return tc::launch(true, norm_kernel<TX, TR, TY, kTeam, kChunks>, dim3((unsigned)((a.n_rows + (long long)kTeams - 1) / kTeams)),
                    dim3(kTeam * kTeams), 0, st, a);
}
template <class TX, class TR, class TY>
cudaError_t launch_norm(const NormArgs& a, cudaStream_t st) {
  const int chunks = (a.width + 7) / 8;
  if (chunks <= 32) return launch_norm<TX, TR, TY, 32, 1>(a, st);
  if (chunks <= 64) return launch_norm<TX, TR, TY, 32, 2>(a, st);
  if (chunks <= 128) return launch_norm<TX, TR, TY, 128, 1>(a, st);
  if (chunks <= 256) return launch_norm<TX, TR, TY, 256, 1>(a, st);
  if (chunks <= 512) return launch_norm<TX, TR, TY, 512, 1>(a, st);
  if (chunks <= 1024) return launch_norm<TX, TR, TY, 512, 2>(a, st);
  return launch_norm<TX, TR, TY, 1024, 2>(a, st);
}
template <class TX, class TR>
cudaError_t launch_norm(const NormArgs& a, int y_dtype, cudaStream_t st) {
  if (y_dtype == MCD_WEIGHT_F32) return launch_norm<TX, TR, float>(a, st);
  if (y_dtype == MCD_WEIGHT_BF16) return launch_norm<TX, TR, uint16_t>(a, st);
  return launch_norm<TX, TR, uint8_t>(a, st);
}
template <class TX>
cudaError_t launch_norm(const NormArgs& a, int res_dtype, int y_dtype, cudaStream_t st) {
  return res_dtype == MCD_WEIGHT_F32 ? launch_norm<TX, float>(a, y_dtype, st) : launch_norm<TX, uint16_t>(a, y_dtype, st);
}

}  // namespace
}  // namespace rows
}  // namespace mcd

using namespace mcd;

extern "C" mcd_status mcd_norm_rows(int32_t n_rows, int32_t width, const void* x, int64_t x_stride, int32_t x_dtype,
                                    const void* residual, int64_t residual_stride, void* sum, int64_t sum_stride,
                                    int32_t res_dtype, int32_t norm, const float* gain, float eps, void* y,
                                    int64_t y_stride, int32_t y_dtype, float* y_scale, void* stream) {
  using namespace rows;
  if (n_rows < 0 || width <= 0) return MCD_ERR_INVALID_ARG;
  const bool k8 = y_dtype == MCD_E4M3;
  auto plain = [](int32_t d) { return d == MCD_WEIGHT_F32 || d == MCD_WEIGHT_BF16; };
  if (!plain(x_dtype) || (!plain(y_dtype) && !k8) || ((residual || sum) && !plain(res_dtype))) return MCD_ERR_UNSUPPORTED;
  if (norm && !(eps >= 0.f && std::isfinite(eps))) return MCD_ERR_INVALID_ARG;
  if (width > 16384) return MCD_ERR_UNSUPPORTED;
  if (n_rows == 0) return MCD_OK;
  if (!x || !y || (k8 && !y_scale)) return MCD_ERR_INVALID_ARG;
  const Block in[2] = {{x, x_stride, n_rows, width, bytes_of(x_dtype)}, {residual, residual_stride, n_rows, width, bytes_of(res_dtype)}};
  const Block out[2] = {{sum, sum_stride, n_rows, width, bytes_of(res_dtype)}, {y, y_stride, n_rows, width, bytes_of(y_dtype)}};
  for (const Block* b : {&in[0], &in[1], &out[0], &out[1]}) {
    if (!b->p) continue;
    if (b->stride < width) return MCD_ERR_INVALID_ARG;
    if (!b->aligned() || !b->fits()) return MCD_ERR_UNSUPPORTED;
  }
  const Block one_gain = values(gain, width, 4), scales = values(k8 ? y_scale : nullptr, n_rows, 4);
  if (!aligned_to(gain, 16) || !aligned_to(scales.p, 4)) return MCD_ERR_UNSUPPORTED;
  for (const Block& o : out) {
    for (const Block& i : in)
      if (overlap(o, i) && !same(o, i)) return MCD_ERR_INVALID_ARG;
    if (overlap(o, one_gain) || overlap(o, scales)) return MCD_ERR_INVALID_ARG;
  }
  if (overlap(out[0], out[1]) || overlap(scales, in[0]) || overlap(scales, in[1]) || overlap(scales, one_gain)) return MCD_ERR_INVALID_ARG;
  const NormArgs a{x, residual, sum, y, gain, y_scale, x_stride, residual_stride, sum_stride, y_stride, n_rows, width, norm, norm ? eps : 0.f,
                   1.f / (float)width};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int res = residual || sum ? res_dtype : MCD_WEIGHT_F32;
  return cuda_status(x_dtype == MCD_WEIGHT_F32 ? launch_norm<float>(a, res, y_dtype, st) : launch_norm<uint16_t>(a, res, y_dtype, st));
}
