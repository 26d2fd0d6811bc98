// Shared by the paged cache's operators (include/mcd_cache.h): views of the page table and of a
// call's rows with their bounds checks, and the host's checks of descriptors.
#pragma once
#include <atomic>
#include <cmath>

#include "mcd_host.cuh"
#include "mcd_tcgemm.cuh"
#include "../../include/mcd_cache.h"

namespace mcd {
namespace paged {

// The first failure stays (err is zeroed by the caller).
__device__ __forceinline__ void report(int* err, mcd_status s) { atomicCAS(err, 0, (int)s); }

// Rows and cached positions of one sequence; n = -1 when its numbers do not fit the call's bounds.
struct Seq {
  int row0, n, cached;
};
__device__ __forceinline__ Seq load_seq(const mcd_chunks& ch, int s) {
  Seq q;
  const int r0 = __ldg(ch.row_start + s), r1 = __ldg(ch.row_start + s + 1);
  q.cached = __ldg(ch.cached + s);
  q.row0 = r0;
  q.n = r1 - r0;
  if (r0 < 0 || r1 < r0 || r1 > ch.n_rows || q.n > ch.max_rows || q.cached < 0 || q.cached > ch.max_tokens - q.n) q.n = -1;
  return q;
}

// The last s in [0, n) with at(s) <= x, for ascending at and at(0) <= x; every lane of the warp
// calls it with the same x.  32 probes a round: two dependent loads for a thousand sequences, where
// halving takes ten.
template <class At>
__device__ __forceinline__ int warp_last_le(int n, At at, long long x) {
  const int lane = threadIdx.x & 31;
  int lo = 0, len = n;                           // the answer is in [lo, lo + len)
  while (len > 1) {
    const int step = (len + 31) / 32, i = lo + lane * step;
    const unsigned m = __ballot_sync(0xffffffffu, lane * step < len && at(i) <= x);
    const int last = m ? 31 - __clz(m) : 0;      // ascending: the set lanes are a prefix
    lo += last * step;
    len = min(step, len - last * step);
  }
  return lo;
}

// Two fp32 operations an instruction.
__device__ __forceinline__ uint64_t pack2(float x, float y) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x), "f"(y));
  return d;
}
__device__ __forceinline__ void unpack2(uint64_t d, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(d)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// ---- host side -------------------------------------------------------------------------------
inline int esize(int dtype) { return dtype == MCD_WEIGHT_F32 ? 4 : 2; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline mcd_status check_kv(const mcd_paged_kv* kv) {
  if (!kv || !kv->k || !kv->v || kv->n_layers <= 0 || kv->n_pages <= 0 || kv->n_kv_heads <= 0) return MCD_ERR_INVALID_ARG;
  if (kv->dtype != MCD_WEIGHT_F32 && kv->dtype != MCD_WEIGHT_BF16) return MCD_ERR_UNSUPPORTED;
  if (kv->head_dim != 64 && kv->head_dim != 128) return MCD_ERR_UNSUPPORTED;
  if (kv->page_size != 16 && kv->page_size != 32 && kv->page_size != 64 && kv->page_size != 128) return MCD_ERR_UNSUPPORTED;
  if (kv->n_kv_heads > 1024) return MCD_ERR_UNSUPPORTED;
  const int per16 = 16 / esize(kv->dtype);
  const int64_t st[4] = {kv->layer_stride, kv->page_stride, kv->head_stride, kv->token_stride};
  for (int64_t s : st)
    if (s < kv->head_dim || s % per16 || s >= (1ll << 37)) return MCD_ERR_UNSUPPORTED;
  if (!aligned16(kv->k) || !aligned16(kv->v)) return MCD_ERR_UNSUPPORTED;
  return MCD_OK;
}

inline mcd_status check_chunks(const mcd_chunks* ch, const mcd_paged_kv* kv) {
  if (!ch || ch->n_seqs < 0 || ch->n_rows < 0 || ch->max_rows < 0 || ch->max_tokens < 0 || ch->table_stride < 0)
    return MCD_ERR_INVALID_ARG;
  if (ch->n_seqs == 0 || ch->n_rows == 0 || ch->max_rows == 0) return MCD_OK;
  if (!ch->table || !ch->cached || !ch->row_start) return MCD_ERR_INVALID_ARG;
  if (ch->max_tokens > (int64_t)ch->table_stride * kv->page_size) return MCD_ERR_INVALID_ARG;
  if (ch->n_seqs > 65535 || ch->n_rows >= (1 << 27)) return MCD_ERR_UNSUPPORTED;
  return MCD_OK;
}
inline bool no_rows(const mcd_chunks* ch) { return ch->n_seqs == 0 || ch->n_rows == 0 || ch->max_rows == 0; }

// SMs of the current device, looked up once per device.
inline int sm_count() {
  static std::atomic<int> known[64];
  int dev = 0, n = 152;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return n;
  const int k = known[dev].load(std::memory_order_relaxed);
  if (k) return k;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

}  // namespace paged
}  // namespace mcd
