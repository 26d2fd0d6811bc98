// Shared by the operators on rows (include/mcd_rows.h): eight elements at a time, joins of a team of threads, and the
// host's checks of what overlaps.
#pragma once
#include "mcd_host.cuh"
#include "mcd_tcgemm.cuh"
#include "../../include/mcd_rows.h"

namespace mcd {
namespace rows {

// The larger one, NaN where either is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Eight values of a type: fp32, bf16 (uint16_t) or e4m3 (uint8_t, stores only).  Rounding is to the nearest, ties to even;
// e4m3 keeps values beyond 448 at 448.
template <class T>
struct Vec8;
template <>
struct Vec8<float> {
  static __device__ __forceinline__ float one(float x) { return x; }
  static __device__ __forceinline__ float round(float x) { return x; }
  static __device__ __forceinline__ void load(const float* p, float (&v)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
};
template <>
struct Vec8<uint16_t> {
  static __device__ __forceinline__ float one(uint16_t x) { return bf16_bits_to_f32(x); }
  static __device__ __forceinline__ uint16_t round(float x) { return (uint16_t)pack_bf16x2(x, 0.f); }
  static __device__ __forceinline__ void load(const uint16_t* p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo_f32(w[i]), v[2 * i + 1] = bf16_hi_f32(w[i]);
  }
  static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) =
        make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  }
};
template <>
struct Vec8<uint8_t> {
  static __device__ __forceinline__ uint32_t pair(float lo, float hi) {
    uint16_t d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(hi), "f"(lo));
    return d;
  }
  static __device__ __forceinline__ uint8_t round(float x) { return (uint8_t)pair(x, 0.f); }
  static __device__ __forceinline__ void store(uint8_t* p, const float (&v)[8]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pair(v[0], v[1]) | pair(v[2], v[3]) << 16, pair(v[4], v[5]) | pair(v[6], v[7]) << 16);
  }
};

// Sum of q and (with kMax) maximum of m >= 0 over a team: a warp, or the whole CTA.  Every thread of the team calls it, once.
// (Bit patterns of numbers that are not negative are in the numbers' order, NaN above all.)
template <int kTeam, bool kMax>
__device__ __forceinline__ void team_join(float& q, float& m) {
#pragma unroll
  for (int w = 16; w; w >>= 1) q += __shfl_xor_sync(0xffffffffu, q, w);
  if (kMax) m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
  if (kTeam > 32) {
    constexpr int kWarps = kTeam / 32;
    __shared__ float2 part[kWarps];
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = make_float2(q, m);
    __syncthreads();
    const float2 p = part[threadIdx.x % kWarps];       // (every warp joins them all, each in the lanes of its kind)
    q = p.x;
#pragma unroll
    for (int w = kWarps / 2; w; w >>= 1) q += __shfl_xor_sync(0xffffffffu, q, w);
    if (kMax) m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(p.y)));
  }
}

// ---- host side -------------------------------------------------------------------------------
inline int bytes_of(int dtype) { return dtype == MCD_WEIGHT_F32 ? 4 : dtype == MCD_WEIGHT_BF16 ? 2 : 1; }

// Rows of `width` elements of `size` bytes, `stride` elements apart.
struct Block {
  const void* p;
  int64_t stride, n_rows, width;
  int size;
  uintptr_t at() const { return reinterpret_cast<uintptr_t>(p); }
  uintptr_t end() const { return at() + (uintptr_t)(((n_rows - 1) * stride + width) * size); }
  bool aligned() const { return !(at() & 15u) && (n_rows < 2 || stride * size % 16 == 0); }
  bool fits() const { return n_rows < 2 || stride <= (1ll << 60) / (n_rows * size); }      // (its bytes can be counted)
};
// n values of `size` bytes one after another (null: none).
inline Block values(const void* p, int64_t n, int size) { return {p, n, 1, n, size}; }
inline bool aligned_to(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline bool same(const Block& a, const Block& b) { return a.p == b.p && a.size == b.size && (a.n_rows < 2 || a.stride == b.stride); }
// Whether two blocks share a byte.  (Rows of one stride may lie beside each other; of two strides that is not looked into.)
inline bool overlap(const Block& a, const Block& b) {
  if (!a.p || !b.p || a.n_rows <= 0 || b.n_rows <= 0 || a.end() <= b.at() || b.end() <= a.at()) return false;
  const uintptr_t step = (uintptr_t)(a.stride * a.size);
  if (a.n_rows < 2 || b.n_rows < 2 || step != (uintptr_t)(b.stride * b.size)) return true;
  const uintptr_t wa = (uintptr_t)(a.width * a.size), wb = (uintptr_t)(b.width * b.size);
  const uintptr_t ahead = (b.at() % step + step - a.at() % step) % step;      // b's rows start so far behind a's
  return ahead < wa || step - ahead < wb;
}

}  // namespace rows
}  // namespace mcd
