// mcd_tc_gemm_e4m3 (include/mcd_tc.h): Y[n][m] = a_scale[m] b_scale[n] sum_k A[m][k] B[n][k] on 8-bit operands.
//
// The products are tcgen05.mma of kind f8f6f4 (K = 32 an instruction): 128 rows of A in the accumulator's lanes, up to 256 rows
// of B in its columns.  Operands come by TMA from the row-major matrices, 128 of K a stage, into rows of 128 swizzled bytes;
// what lies behind the matrices' ends is read as zeros.
// What bounds it: many rows the tensor cores (8,192 x 8,192 x 8,192: 304 us, 3.6 PFLOP/s; 6,144 x 8,191 x 4,096: 115 us alone, 134 in a
// row of such calls at the power limit, tensor pipe 89 % active; one CTA a tile of 128 x 256: 438 and 183); few rows the stream of A
// (6,144 x 4 x 4,096: 7.9 us, 3.2 TB/s; 131,072 x 4 x 4,096: 85 us, 6.3 TB/s) and, below about 4 us, the start of a kernel.
#include <cooperative_groups.h>

#include <algorithm>

#include "mcd_attn.cuh"
#include "mcd_rows.cuh"
#include "../../include/mcd_tc.h"

namespace mcd {
namespace tc {
namespace {

namespace cg = cooperative_groups;

constexpr int kK8 = 128;               // of K a stage: one swizzled row
constexpr unsigned long long kWait8 = 2000000000ull;

struct Args8 {
  const float *a_scale, *b_scale;
  void* y;
  long long ldy;
  int M, N, K;
  int pitch, splits, deep;             // rows of B a tile, parts of K, Layout8's kDeep
  int* err;
};

// Instruction descriptor: e4m3 A and B (K-major), fp32 D.
__host__ __device__ constexpr uint32_t idesc_e4m3(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void umma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
// Box of 128 bytes of K from k on, rows from `row` on.
__device__ __forceinline__ void tma_rows8(void* dst, const CUtensorMap* map, int k, int row, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
      "l"(map), "r"(k), "r"(row), "r"(smem_u32(bar))
      : "memory");
}

// Columns (rows n0 .. of Y) of an accumulator to Y: 32 at a time from tensor memory, scaled, rounded, laid out as rows of 128
// in shared memory and stored by TMA, 16 rows a box.  Two chunks have room, `turn` is the next one's: one is stored while the other
// is written.  Four warps call it together (w: the warp's quarter of the lanes); before the CTA ends, drain_done.  (Stored from registers, 64 bytes of a
// row at a time, a tile of 256 columns took 12 us.)
constexpr int kChunkCols = 32;
template <class T>
__host__ __device__ constexpr int chunk_bytes() { return kChunkCols * kBM * (int)sizeof(T); }
template <class T>
__device__ __forceinline__ void drain(const Args8& g, const CUtensorMap* y_map, uint8_t* room, uint32_t& turn, uint32_t tmem, int n0, int live, int m0, int w) {
  const int lane = threadIdx.x & 31, r = w * 32 + lane, m = m0 + r;
  const float sa = g.a_scale && m < g.M ? __ldg(g.a_scale + m) : 1.f;
  const uint32_t lanes = tmem + ((uint32_t)(w * 32) << 16);
  // (a box that is cut inside 16 bytes is written up to their end, over what is not Y's: such a tile is stored by elements)
  const bool ragged = m0 + kBM > g.M && g.M % (16 / (int)sizeof(T)) != 0;
  for (int c = 0; c < live; c += kChunkCols, turn ^= 1) {
    uint32_t x[32];
    paged::tmem_ld32(lanes + c, x);
    const float sb = g.b_scale && c + lane < live ? __ldg(g.b_scale + n0 + c + lane) : 1.f;
    paged::tmem_loaded(x);
    T v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = rows::Vec8<T>::round(__uint_as_float(x[j]) * sa * __shfl_sync(0xffffffffu, sb, j));
    if (ragged) {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (c + j < live && m < g.M) static_cast<T*>(g.y)[(n0 + c + j) * g.ldy + m] = v[j];
      __syncwarp();
      continue;
    }
    T* const place = reinterpret_cast<T*>(room + turn * chunk_bytes<T>());
#pragma unroll
    for (int j = 0; j < 32; ++j) place[j * kBM + r] = v[j];
    // (the chunk before has been read when the next is written)
    if (w == 0 && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();                                      // (barriers and loads of tensor memory want a warp together)
    fence_proxy_async();
    asm volatile("bar.sync 1, 128;" ::: "memory");
    if (w == 0 && lane == 0) {
      for (int b = 0; b < min(kChunkCols, live - c); b += 16)
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(y_map), "r"(m0), "r"(n0 + c + b),
                     "r"(smem_u32(place + b * kBM))
                     : "memory");
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    __syncwarp();
  }
}
// (of the thread that issued the stores: they are done)
__device__ __forceinline__ void drain_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// Four neighbours of row n.
template <class T>
__device__ __forceinline__ void store4_scaled(const Args8& g, int n, int m, float4 v) {
  const float sb = g.b_scale ? __ldg(g.b_scale + n) : 1.f;
  float x[4] = {v.x, v.y, v.z, v.w};
  // (a's scale, then b's, as drain does it: their product may leave fp32's range where the result does not)
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = x[e] * (g.a_scale && m + e < g.M ? __ldg(g.a_scale + m + e) : 1.f) * sb;
  T* y = static_cast<T*>(g.y) + n * g.ldy + m;
  if (m + 4 <= g.M) {
    paged::store4(y, make_float4(x[0], x[1], x[2], x[3]));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (m + e < g.M) y[e] = rows::Vec8<T>::round(x[e]);
  }
}

// kDeep: a ring that fills an SM; without, two CTAs share one (up to 128 columns).
template <int BN, bool kDeep>
struct Layout8 {
  static constexpr int kABytes = kBM * kK8, kStageBytes = kABytes + BN * kK8;
  static constexpr int kStages = kDeep ? (kStageBudget / kStageBytes > 8 ? 8 : kStageBudget / kStageBytes) : BN <= 64 ? 4 : 3;
  static constexpr int kBar = kStages * kStageBytes;                   // full[s], empty[s], accum
  static constexpr int kMisc = kBar + (2 * kStages + 1) * 8;            // tensor memory address, abort
  static constexpr int kBytes = kMisc + 8 + 1024;                       // + alignment
  static constexpr int kCols = tmem_cols_for(BN);
  static constexpr int kPitch = kBM + 4;                                // floats of a row of partial sums
  static_assert(BN * kPitch * 4 <= kBar && 2 * chunk_bytes<float>() <= kBar && kBytes <= 227 * 1024, "results take the stages' place");
};

// A tile of 128 x pitch per CTA over a part of K; the parts' CTAs are a cluster and add up through shared memory, in the
// order of the parts.  Warp 0 copies, warp 1 multiplies, warps 2 to 5 store.
constexpr int kThreads8 = 192, kMaxParts = 8;
template <class T, int BN, bool kDeep>
__global__ void __launch_bounds__(kThreads8, 1)
    gemm8_tile_kernel(const Args8 g, const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                      const __grid_constant__ CUtensorMap y_map) {
  using L = Layout8<BN, kDeep>;
  constexpr int S = L::kStages;
  extern __shared__ uint8_t g8_smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(g8_smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBar);
  uint64_t *empty = full + S, *accum = empty + S;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::kMisc + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int part = blockIdx.x % g.splits, m0 = (int)(blockIdx.x / g.splits) * kBM, n0 = blockIdx.y * g.pitch;
  const int nk_all = (g.K + kK8 - 1) / kK8, per = (nk_all + g.splits - 1) / g.splits;
  const int k0 = part * per, nk = min(nk_all, k0 + per) - k0;
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    mbar_init(accum, 1);
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async();
    asm volatile("prefetch.tensormap [%0];" ::"l"(&a_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&b_map) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)L::kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  pdl_trigger();
  if (warp == 0) {
    if (lane == 0) {
      int i = 0;
      const uint32_t bytes = L::kABytes + g.pitch * kK8;
      for (; i < nk; ++i) {
        const int s = i % S;
        if (i >= S && !tc_wait(&empty[s], (i / S - 1) & 1, g.err, kWait8)) *abort_flag = 1;
        if (*abort_flag) break;
        mbar_arrive_expect_tx(&full[s], bytes);
        tma_rows8(smem + s * L::kStageBytes, &a_map, (k0 + i) * kK8, m0, &full[s]);
        tma_rows8(smem + s * L::kStageBytes + L::kABytes, &b_map, (k0 + i) * kK8, n0, &full[s]);
      }
      // every copy lands before its place is used again
      for (int n = max(0, i - S); n < i; ++n) tc_wait(&full[n % S], n / S & 1, g.err, kWait8);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = idesc_e4m3(kBM, g.pitch);
      for (int i = 0; i < nk; ++i) {
        const int s = i % S;
        if (!tc_wait(&full[s], i / S & 1, g.err, kWait8)) *abort_flag = 1;
        if (*abort_flag) break;
        tc_fence_after();
        const uint64_t a = sw128_desc(smem_u32(smem + s * L::kStageBytes)), b = sw128_desc(smem_u32(smem + s * L::kStageBytes + L::kABytes));
#pragma unroll
        for (int j = 0; j < kK8 / 32; ++j) umma_e4m3(tmem, a + 2 * j, b + 2 * j, idesc, (i | j) != 0);
        umma_commit(&empty[s]);
      }
      umma_commit(accum);
    }
    __syncwarp();
  }
  const bool ok = __syncthreads_and(paged::warp_wait(accum, 0, g.err, abort_flag));      // (copies are done too)
  tc_fence_after();
  const int quarter = warp & 3, r = quarter * 32 + lane;
  const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
  const int live = min(g.pitch, g.N - n0);
  if (g.splits == 1) {
    if (warp >= 2 && ok) {
      uint32_t turn = 0;
      drain<T>(g, &y_map, smem, turn, tmem, n0, live, m0, quarter);
      if (quarter == 0 && lane == 0) drain_done();
      __syncwarp();
    }
  } else {
    cg::cluster_group cl = cg::this_cluster();
    float* sums = reinterpret_cast<float*>(smem);
    if (warp >= 2) {
      for (int c = 0; c < live; c += 16) {
        float v[16];
        tmem_ld16(lanes + c, v);
#pragma unroll
        for (int j = 0; j < 16; ++j) sums[(c + j) * L::kPitch + r] = v[j];
      }
    }
    cl.sync();
    const float* from[kMaxParts];
#pragma unroll
    for (int z = 0; z < kMaxParts; ++z) from[z] = cl.map_shared_rank(sums, min(z, g.splits - 1)) + 4 * lane;
    // a warp has a column, a lane four rows of it
    for (int c = part + g.splits * warp; c < live; c += g.splits * (kThreads8 / 32)) {
      float4 x[kMaxParts];
#pragma unroll
      for (int z = 0; z < kMaxParts; ++z)
        if (z < g.splits) x[z] = *reinterpret_cast<const float4*>(from[z] + c * L::kPitch);
      float4 v = x[0];
#pragma unroll
      for (int z = 1; z < kMaxParts; ++z)
        if (z < g.splits) v.x += x[z].x, v.y += x[z].y, v.z += x[z].z, v.w += x[z].w;
      if (m0 + 4 * lane < g.M) store4_scaled<T>(g, n0 + c, m0 + 4 * lane, v);
    }
    __syncwarp();
    cl.sync();                                         // nobody leaves while others read
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)L::kCols) : "memory");
  }
}

// Tiles of 256 x 256 by pairs of CTAs, each with an SM: CTA r holds 128 of the tile's rows of A and 128 of B, the products
// (tcgen05.mma of the pair) read both CTAs' and leave 128 x 256 in either's tensor memory.  The operands that an SM reads for a
// product halve against 128 x 256 alone.  The pairs stay and go from tile to tile, the copies ahead of the products through
// six stages, the products of a tile under the stores of the one before (two accumulators).
//   warp 0 of either CTA      copies its rows; their bytes complete the first CTA's barrier
//   warp 1 of the first CTA   products; a stage is given back to both CTAs
//   warps 2 to 5 of either    stores
constexpr int kPairTile = 256;
struct PairLayout8 {
  static constexpr int kStages = 6, kStageBytes = 2 * kBM * kK8;
  static constexpr int kRoom = kStages * kStageBytes;                  // two chunks of results
  static constexpr int kBar = kRoom + 2 * chunk_bytes<float>();         // full[S] empty[S] acc_full[2] acc_empty[2]
  static constexpr int kMisc = kBar + (2 * kStages + 4) * 8;
  static constexpr int kBytes = kMisc + 8 + 1024;
  static_assert(kBytes <= 227 * 1024, "shared memory");
};
__device__ __forceinline__ uint32_t of_rank(uint32_t addr, uint32_t rank) {
  uint32_t d;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"(addr), "r"(rank));
  return d;
}
__device__ __forceinline__ void umma_e4m3_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
// Arrives at the barrier of this place in both CTAs once the products issued so far are done.
__device__ __forceinline__ void umma_commit_pair(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((uint16_t)3)
               : "memory");
}
// As tma_rows8, completing a barrier of the pair's first CTA.
__device__ __forceinline__ void tma_rows8_pair(void* dst, const CUtensorMap* map, int k, int row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(
          smem_u32(dst)),
      "l"(map), "r"(k), "r"(row), "r"(bar)
      : "memory");
}

template <class T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads8, 1)
    gemm8_pair_kernel(const Args8 g, const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                      const __grid_constant__ CUtensorMap y_map) {
  using L = PairLayout8;
  constexpr int S = L::kStages;
  extern __shared__ uint8_t g8_smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(g8_smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBar);
  uint64_t *empty = full + S, *acc_full = empty + S, *acc_empty = acc_full + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::kMisc + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  cg::cluster_group cl = cg::this_cluster();
  const uint32_t rank = cl.block_rank();
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 8);                     // the storing warps of both CTAs
    }
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async();
    asm volatile("prefetch.tensormap [%0];" ::"l"(&a_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&b_map) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  cl.sync();                                           // (barriers and tensor memory of both)
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  pdl_trigger();
  const int m_tiles = (g.M + kPairTile - 1) / kPairTile, n_tiles = (g.N + kPairTile - 1) / kPairTile;
  const int nk = (g.K + kK8 - 1) / kK8, step = (int)gridDim.x / 2, first = (int)blockIdx.x / 2;
  const long long tiles = (long long)m_tiles * n_tiles;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t i = 0;
      for (long long t = first; t < tiles && !*abort_flag; t += step) {
        const int m0 = (int)(t % m_tiles) * kPairTile + (int)rank * kBM, n0 = (int)(t / m_tiles) * kPairTile + (int)rank * kBM;
        for (int k = 0; k < nk; ++k, ++i) {
          const uint32_t s = i % S;
          if (i >= (uint32_t)S && !tc_wait(&empty[s], (i / S - 1) & 1, g.err, kWait8)) *abort_flag = 1;
          if (*abort_flag) break;
          const uint32_t bar = of_rank(smem_u32(&full[s]), 0);
          if (rank == 0) mbar_arrive_expect_tx(&full[s], 2 * L::kStageBytes);
          tma_rows8_pair(smem + s * L::kStageBytes, &a_map, k * kK8, m0, bar);
          tma_rows8_pair(smem + s * L::kStageBytes + kBM * kK8, &b_map, k * kK8, n0, bar);
        }
      }
      // every copy of either CTA lands before the pair may end
      if (rank == 0)
        for (uint32_t n = i > (uint32_t)S ? i - S : 0u; n < i; ++n) tc_wait(&full[n % S], n / S & 1, g.err, kWait8);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      // the whole warp runs along, one elected lane issues
      constexpr uint32_t idesc = idesc_e4m3(kPairTile, kPairTile);
      const uint64_t a0 = sw128_desc(smem_u32(smem)), b0 = sw128_desc(smem_u32(smem + kBM * kK8));
      uint32_t s = 0, phase = 0;
      int n = 0;
      bool ok = true;
      for (long long t = first; t < tiles && ok; t += step, ++n) {
        const int buf = n & 1;
        if (n >= 2) ok = paged::warp_wait(&acc_empty[buf], (n / 2 - 1) & 1, g.err, abort_flag);
        if (!ok) break;
        tc_fence_after();
        const uint32_t d = tmem + buf * kPairTile;
        for (int k = 0; k < nk; ++k) {
          ok = paged::warp_wait(&full[s], phase, g.err, abort_flag);
          if (!ok) break;
          tc_fence_after();
          if (paged::elect_one()) {
            const uint64_t at = s * (uint64_t)(L::kStageBytes >> 4);
#pragma unroll
            for (int j = 0; j < kK8 / 32; ++j) umma_e4m3_pair(d, a0 + at + 2 * j, b0 + at + 2 * j, idesc, (k | j) != 0);
            umma_commit_pair(&empty[s]);
          }
          __syncwarp();
          if (++s == S) s = 0, phase ^= 1;
        }
        if (paged::elect_one()) umma_commit_pair(&acc_full[buf]);
        __syncwarp();
      }
    }
  } else {
    const int quarter = warp & 3;
    int n = 0;
    uint32_t turn = 0;
    bool ok = true;
    for (long long t = first; t < tiles; t += step, ++n) {
      const int buf = n & 1, m0 = (int)(t % m_tiles) * kPairTile + (int)rank * kBM, n0 = (int)(t / m_tiles) * kPairTile;
      // (the four warps decide alike: they meet in drain)
      ok = paged::warp_wait(&acc_full[buf], n / 2 & 1, g.err, abort_flag);
      uint32_t all;
      asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.and.pred q, 2, 128, p;\n selp.u32 %0, 1, 0, q;\n}\n" : "=r"(all) : "r"((uint32_t)ok) : "memory");
      if (!all) break;
      tc_fence_after();
      if (m0 < g.M) drain<T>(g, &y_map, smem + L::kRoom, turn, tmem + buf * kPairTile, n0, min(kPairTile, g.N - n0), m0, quarter);
      tc_fence_before();
      __syncwarp();
      if (lane == 0)
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(of_rank(smem_u32(&acc_empty[buf]), 0)) : "memory");
      __syncwarp();
    }
    if (quarter == 0 && lane == 0) drain_done();
    __syncwarp();
  }
  tc_fence_before();
  cl.sync();                                           // products, copies and stores of both are done
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// Tensor map of a row-major 8-bit matrix, boxes of `box` rows and 128 of K.
bool map8(CUtensorMap* map, const void* p, int rows, int K, long long ld, int box) {
  const paged::EncodeTiled encode = paged::tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  const cuuint32_t boxes[2] = {kK8, (cuuint32_t)box}, one[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, boxes, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tensor map of Y, boxes of 16 rows and 128 elements.
template <class T>
bool map_y(CUtensorMap* map, const Args8& g) {
  const paged::EncodeTiled encode = paged::tensor_map_encoder();
  if (!encode) return false;
  const long long ld = g.N > 1 ? g.ldy : ((long long)g.M + 7) / 8 * 8;
  const cuuint64_t dims[2] = {(cuuint64_t)g.M, (cuuint64_t)g.N}, strides[1] = {(cuuint64_t)(ld * (long long)sizeof(T))};
  const cuuint32_t boxes[2] = {kBM, 16}, one[2] = {1, 1};
  return encode(map, sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, g.y, dims, strides, boxes, one,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T, int BN, bool kDeep>
cudaError_t launch_tile8(const Args8& g, const CUtensorMap& a_map, const CUtensorMap& b_map, const CUtensorMap& y_map, cudaStream_t st) {
  static std::atomic<unsigned> done{0};
  using L = Layout8<BN, kDeep>;
  cudaError_t e = paged::opt_in(gemm8_tile_kernel<T, BN, kDeep>, L::kBytes, done);
  if (e != cudaSuccess) return e;
  return paged::launch_clusters(gemm8_tile_kernel<T, BN, kDeep>, dim3((g.M + kBM - 1) / kBM * g.splits, (g.N + g.pitch - 1) / g.pitch), kThreads8,
                                g.splits, L::kBytes, st, g, a_map, b_map, y_map);
}
template <class T>
cudaError_t launch_tile8(const Args8& g, bool deep, const CUtensorMap& a_map, const CUtensorMap& b_map, const CUtensorMap& y_map, cudaStream_t st) {
  if (g.pitch <= 32) return deep ? launch_tile8<T, 32, true>(g, a_map, b_map, y_map, st) : launch_tile8<T, 32, false>(g, a_map, b_map, y_map, st);
  if (g.pitch <= 64) return deep ? launch_tile8<T, 64, true>(g, a_map, b_map, y_map, st) : launch_tile8<T, 64, false>(g, a_map, b_map, y_map, st);
  if (g.pitch <= 128) return deep ? launch_tile8<T, 128, true>(g, a_map, b_map, y_map, st) : launch_tile8<T, 128, false>(g, a_map, b_map, y_map, st);
  return launch_tile8<T, 256, true>(g, a_map, b_map, y_map, st);
}

// Pairs that run at a time, looked up once per device.
template <class T>
int pair_count() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 1;
  if (const int k = known[dev].load(std::memory_order_relaxed)) return k;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * (unsigned)paged::sm_count());
  cfg.blockDim = dim3(kThreads8);
  cfg.dynamicSmemBytes = PairLayout8::kBytes;
  if (cudaOccupancyMaxActiveClusters(&n, gemm8_pair_kernel<T>, &cfg) != cudaSuccess || n < 1) return 1;
  known[dev].store(n, std::memory_order_relaxed);
  return n;
}
template <class T>
cudaError_t launch_pair8(const Args8& g, const CUtensorMap& a_map, const CUtensorMap& b_map, const CUtensorMap& y_map, cudaStream_t st) {
  static std::atomic<unsigned> done{0};
  cudaError_t e = paged::opt_in(gemm8_pair_kernel<T>, PairLayout8::kBytes, done);
  if (e != cudaSuccess) return e;
  const long long tiles = (long long)((g.M + kPairTile - 1) / kPairTile) * ((g.N + kPairTile - 1) / kPairTile);
  const int pairs = (int)std::min<long long>(tiles, pair_count<T>());
  return launch(true, gemm8_pair_kernel<T>, dim3(2 * pairs), dim3(kThreads8), PairLayout8::kBytes, st, g, a_map, b_map, y_map);
}

// Rows of B a tile and parts of K, by what they were measured to cost (us; 6144, 4096, 2048 and 1024 rows of A, K of 1024 to
// 4096, 1 to 2048 rows of B): a CTA starts and ends in about 3, a slice of 128 of K takes 0.25 where a CTA has an SM to itself
// and 0.35 where two share one, a little more with wide tiles, its columns 0.012 each to store; parts are joined in
// 0.2 + 0.035 a column.  6144 x 4 x 1024: one part 4.7, four 3.9; 6144 x 128 x 1024: one 5.6, two 7.1.  More than four
// thirds of the SMs' clusters do not run at a time, nor do clusters of eight that want an SM a CTA on more than half of them (2048 x 4
// x 1024: 6.7, with two CTAs an SM 3.4).
void plan8(Args8& g, int m_tiles, int nk, int n_sm) {
  float best = 0.f;
  const int rows = (g.N + 15) / 16 * 16;
  for (int pitch : {16, 32, 64, 96, 128, 176, 256}) {
    if (pitch > rows && pitch > 16) pitch = rows;
    const long long tiles = (long long)m_tiles * ((g.N + pitch - 1) / pitch);
    for (int s = 1; s <= std::min(kMaxParts, nk); s *= 2) {
      const int per = (nk + s - 1) / s;
      const long long ctas = tiles * s;
      if ((nk + per - 1) / per != s || (s > 1 && 3 * ctas > 4 * n_sm)) continue;
      const bool deep = pitch > 128 || ctas <= (s == 8 ? n_sm / 2 : n_sm);
      const float waves = (float)((ctas + (deep ? 1 : 2) * n_sm - 1) / ((deep ? 1 : 2) * n_sm));
      const float cost = waves * (3.f + per * (deep ? 0.25f : 0.35f) * (1.f + pitch / 512.f) + pitch * 0.012f) + (s > 1 ? 0.2f + 0.035f * pitch : 0.f);
      if (best == 0.f || cost < best) best = cost, g.pitch = pitch, g.splits = s, g.deep = deep;
    }
    if (pitch == rows) break;
  }
}

template <class T>
cudaError_t launch8(Args8 g, const void* A, long long lda, const void* B, long long ldb, cudaStream_t st) {
  const int m_tiles = (g.M + kBM - 1) / kBM, nk = (g.K + kK8 - 1) / kK8, n_sm = paged::sm_count();
  const long long pair_tiles = (long long)((g.M + kPairTile - 1) / kPairTile) * ((g.N + kPairTile - 1) / kPairTile);
  CUtensorMap a_map, b_map, y_map;
  if (!map_y<T>(&y_map, g)) return cudaErrorInvalidValue;
  // Pairs where their tiles fill the SMs, unless few rows of B would fill a quarter of a tile at most (us, pairs against tiles of 128: 20,000 x
  // 1 x 4,096 27.5 and 17.0, x 64 25.7 and 18.2; 131,072 x 4 x 1,024 41.3 and 28.9, x 64 33.4 and 32.8, x 128 36.8 and 39.6, x 256 as fast).
  if (pair_tiles >= n_sm / 2 && g.N > 64) {
    if (!map8(&a_map, A, g.M, g.K, lda, kBM) || !map8(&b_map, B, g.N, g.K, ldb, kBM)) return cudaErrorInvalidValue;
    return launch_pair8<T>(g, a_map, b_map, y_map, st);
  }
  plan8(g, m_tiles, nk, n_sm);
  if (!map8(&a_map, A, g.M, g.K, lda, kBM) || !map8(&b_map, B, g.N, g.K, ldb, g.pitch)) return cudaErrorInvalidValue;
  return launch_tile8<T>(g, g.deep, a_map, b_map, y_map, st);
}

}  // namespace
}  // namespace tc
}  // namespace mcd

using namespace mcd;

extern "C" mcd_status mcd_tc_gemm_e4m3(int32_t M, int32_t N, int32_t K, const void* A, int64_t lda, const float* a_scale,
                                       const void* B, int64_t ldb, const float* b_scale, void* Y, int64_t ldy,
                                       int32_t y_dtype, int32_t* err, void* stream) {
  if (M < 0 || N < 0 || K < 0 || !err) return MCD_ERR_INVALID_ARG;
  if (y_dtype != MCD_WEIGHT_F32 && y_dtype != MCD_WEIGHT_BF16) return MCD_ERR_UNSUPPORTED;
  if (M == 0 || N == 0) return MCD_OK;
  if (!A || !B || !Y || K == 0 || lda < K || ldb < K || ldy < M) return MCD_ERR_INVALID_ARG;
  // (65,535 tiles along N; counts of bytes and of tiles in 32 bits)
  if (M > (1 << 24) || N > (1 << 24) || K > (1 << 24) || lda >= (1ll << 36) || ldb >= (1ll << 36) || ldy >= (1ll << 36))
    return MCD_ERR_UNSUPPORTED;
  const rows::Block a{A, lda, M, K, 1}, b{B, ldb, N, K, 1}, y{Y, ldy, N, M, rows::bytes_of(y_dtype)};
  if (!a.aligned() || !b.aligned() || !y.aligned()) return MCD_ERR_UNSUPPORTED;
  if (!rows::aligned_to(a_scale, 4) || !rows::aligned_to(b_scale, 4) || !rows::aligned_to(err, 4)) return MCD_ERR_UNSUPPORTED;
  const rows::Block sa = rows::values(a_scale, M, 4), sb = rows::values(b_scale, N, 4), e = rows::values(err, 1, 4);
  for (const rows::Block* x : {&a, &b, &sa, &sb})
    if (rows::overlap(y, *x) || rows::overlap(e, *x)) return MCD_ERR_INVALID_ARG;
  if (rows::overlap(y, e)) return MCD_ERR_INVALID_ARG;
  const tc::Args8 g{a_scale, b_scale, Y, ldy, M, N, K, 0, 1, 0, err};
  // (a single row's stride is not looked at: the map wants one all the same)
  const int64_t la = M > 1 ? lda : (K + 15) / 16 * 16, lb = N > 1 ? ldb : (K + 15) / 16 * 16;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return cuda_status(y_dtype == MCD_WEIGHT_F32 ? tc::launch8<float>(g, A, la, B, lb, st) : tc::launch8<uint16_t>(g, A, la, B, lb, st));
}
