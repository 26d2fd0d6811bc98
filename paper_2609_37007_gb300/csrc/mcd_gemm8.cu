// mcd_tc_gemm_e4m3 (include/mcd_tc.h): Y[n][m] = a_scale[m] b_scale[n] sum_k A[m][k] B[n][k] on 8-bit operands.
//
// The products are tcgen05.mma of kind f8f6f4 (K = 32 an instruction): 128 rows of A in the accumulator's lanes, up to 256 rows
// of B in its columns.  Operands come by TMA from the row-major matrices, 128 of K a stage, into rows of 128 swizzled bytes;
// what lies behind the matrices' ends is read as zeros.
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
  int pitch, splits;                   // rows of B a tile, parts of K
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

template <class T>
__device__ __forceinline__ T rounded(float x);
template <>
__device__ __forceinline__ float rounded(float x) { return x; }
template <>
__device__ __forceinline__ uint16_t rounded(float x) { return (uint16_t)pack_bf16x2(x, 0.f); }

template <int BN>
struct Layout8 {
  static constexpr int kABytes = kBM * kK8, kStageBytes = kABytes + BN * kK8;
  static constexpr int kStages = kStageBudget / kStageBytes > 8 ? 8 : kStageBudget / kStageBytes;
  static constexpr int kBar = kStages * kStageBytes;                   // full[s], empty[s], accum
  static constexpr int kMisc = kBar + (2 * kStages + 1) * 8;            // tensor memory address, abort
  static constexpr int kBytes = kMisc + 8 + 1024;                       // + alignment
  static constexpr int kCols = tmem_cols_for(BN);
  static constexpr int kPitch = kBM + 4;                                // floats of a row of partial sums
  static_assert(BN * kPitch * 4 <= kBar && kBytes <= 227 * 1024, "the partial sums take the stages' place");
};

// A tile of 128 x pitch per CTA over a part of K; the parts' CTAs are a cluster and add up through shared memory, in the
// order of the parts.  Warp 0 copies, warp 1 multiplies, warps 2 to 5 store.
constexpr int kThreads8 = 192;
template <class T, int BN>
__global__ void __launch_bounds__(kThreads8, 1)
    gemm8_tile_kernel(const Args8 g, const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map) {
  using L = Layout8<BN>;
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
  const bool ok = tc_wait(accum, 0, g.err, kWait8);
  __syncthreads();                                     // (copies are done too)
  tc_fence_after();
  const int quarter = warp & 3, r = quarter * 32 + lane, m = m0 + r;
  const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
  const float sa = g.a_scale && m < g.M ? __ldg(g.a_scale + m) : 1.f;
  T* const y = static_cast<T*>(g.y);
  const int live = min(g.pitch, g.N - n0);
  if (g.splits == 1) {
    if (warp >= 2 && ok) {
      for (int c = 0; c < live; c += 16) {
        float v[16];
        tmem_ld16(lanes + c, v);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int n = n0 + c + j;
          if (c + j < live && m < g.M) y[n * g.ldy + m] = rounded<T>(v[j] * sa * (g.b_scale ? __ldg(g.b_scale + n) : 1.f));
        }
      }
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
    if (warp >= 2) {
      for (int c = part; c < live; c += g.splits) {
        float v = 0.f;
        for (int z = 0; z < g.splits; ++z) v += *cl.map_shared_rank(sums + c * L::kPitch + r, z);
        const int n = n0 + c;
        if (m < g.M) y[n * g.ldy + m] = rounded<T>(v * sa * (g.b_scale ? __ldg(g.b_scale + n) : 1.f));
      }
    }
    cl.sync();                                         // nobody leaves while others read
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)L::kCols) : "memory");
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

template <class T, int BN>
cudaError_t launch_tile8(const Args8& g, const CUtensorMap& a_map, const CUtensorMap& b_map, cudaStream_t st) {
  static std::atomic<unsigned> done{0};
  cudaError_t e = paged::opt_in(gemm8_tile_kernel<T, BN>, Layout8<BN>::kBytes, done);
  if (e != cudaSuccess) return e;
  return paged::launch_clusters(gemm8_tile_kernel<T, BN>, dim3((g.M + kBM - 1) / kBM * g.splits, (g.N + g.pitch - 1) / g.pitch), kThreads8, g.splits,
                                Layout8<BN>::kBytes, st, g, a_map, b_map);
}

template <class T>
cudaError_t launch8(Args8 g, const void* A, long long lda, const void* B, long long ldb, cudaStream_t st) {
  const int m_tiles = (g.M + kBM - 1) / kBM, nk = (g.K + kK8 - 1) / kK8, n_sm = paged::sm_count();
  const int n_tiles = (g.N + 255) / 256;
  g.pitch = ((g.N + n_tiles - 1) / n_tiles + 15) / 16 * 16;
  g.splits = std::max(1, std::min({8, nk, n_sm / (m_tiles * n_tiles)}));
  const int per = (nk + g.splits - 1) / g.splits;
  g.splits = (nk + per - 1) / per;                     // (no part is empty)
  CUtensorMap a_map, b_map;
  if (!map8(&a_map, A, g.M, g.K, lda, kBM) || !map8(&b_map, B, g.N, g.K, ldb, g.pitch)) return cudaErrorInvalidValue;
  if (g.pitch <= 32) return launch_tile8<T, 32>(g, a_map, b_map, st);
  if (g.pitch <= 64) return launch_tile8<T, 64>(g, a_map, b_map, st);
  if (g.pitch <= 128) return launch_tile8<T, 128>(g, a_map, b_map, st);
  return launch_tile8<T, 256>(g, a_map, b_map, st);
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
  if (M > (1 << 24) || N > (1 << 24) || K > (1 << 24) || lda >= (1ll << 40) || ldb >= (1ll << 40)) return MCD_ERR_UNSUPPORTED;
  const rows::Block a{A, lda, M, K, 1}, b{B, ldb, N, K, 1}, y{Y, ldy, N, M, rows::bytes_of(y_dtype)};
  if (!a.aligned() || !b.aligned() || !y.aligned()) return MCD_ERR_UNSUPPORTED;
  const rows::Block sa{a_scale, M, 1, M, 4}, sb{b_scale, N, 1, N, 4};
  for (const rows::Block* x : {&a, &b, &sa, &sb})
    if (rows::overlap(y, *x)) return MCD_ERR_INVALID_ARG;
  const tc::Args8 g{a_scale, b_scale, Y, ldy, M, N, K, 0, 1, err};
  // (a single row's stride is not looked at: the map wants one all the same)
  const int64_t la = M > 1 ? lda : (K + 15) / 16 * 16, lb = N > 1 ? ldb : (K + 15) / 16 * 16;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return cuda_status(y_dtype == MCD_WEIGHT_F32 ? tc::launch8<float>(g, A, la, B, lb, st) : tc::launch8<uint16_t>(g, A, la, B, lb, st));
}
