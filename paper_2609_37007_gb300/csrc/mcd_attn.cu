// mcd_paged_attention (include/mcd_cache.h): fp32 caches, and bf16 ones with up to 16 query vectors of a
// KV head (the mathematics: mcd_attn.cuh; longer chunks: mcd_attn_chunk.cu).
//
// Both are built to read K and V once.  128 single rows over 17 to 1,023 keys: 50.7 us, 5.2 TB/s (fp32: 205 us, 2.6 TB/s);
// 4 x 2 to 4 rows over up to 120,000: 247 us, 6.2 TB/s of 6.8 measured for a copy.  fp32 chunks: 68.6 us for 24 sequences of 1
// to 200 rows over up to 600 (4 heads of 64), a sixth of the fp32 rate: tiles of 64 rows and 64 keys are half empty, and 16
// warps an SM (their registers) issue every other cycle (packed products, half the instructions: the same time).
#include <algorithm>

#include "mcd_attn.cuh"

namespace mcd {
namespace paged {
namespace {

// ---- plain fp32 arithmetic -------------------------------------------------------------------------
// A CTA of 16 x 16 threads takes 16 RM packed vectors against tiles of 64 keys: thread (ty, tx) has rows
// ty RM .. and keys tx + 16 c of the scores, then dimensions 4 tx .. (+ 64) of the same rows of o.
// The probabilities pass between the 16 threads of a row through shared memory.
constexpr int kFN = 64;
constexpr int kFThreads = 256;

template <int D, int RM>
struct FSmem {
  float q[16 * RM][D + 4], k[kFN][D + 4], v[kFN][D], p[16 * RM][kFN + 4], m[16 * RM], l[16 * RM];
};

template <int D, int RM>
__global__ void __launch_bounds__(kFThreads, 128 / D + (RM == 1)) attn_f32_kernel(const AttnArgs a) {
  extern __shared__ __align__(16) uint8_t f_smem[];
  FSmem<D, RM>& sm = *reinterpret_cast<FSmem<D, RM>*>(f_smem);
  constexpr int kBM = 16 * RM, kDC = D / 64;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int h = blockIdx.y;
  tc::pdl_wait();
  tc::pdl_trigger();
  const int s = a.ranked ? by_tokens(a.ch, blockIdx.z) : blockIdx.z;
  const Seq q = load_seq(a.ch, s);
  if (q.n < 0 && blockIdx.x == 0 && h == 0 && threadIdx.x == 0) report(a.err, MCD_ERR_INVALID_ARG);
  const int z = blockIdx.x % a.splits;
  // (the last tiles see most keys: they come first)
  const int vecs = max(q.n, 0) * a.group, p0 = (gridDim.x / a.splits - 1 - blockIdx.x / a.splits) * kBM;
  if (p0 >= vecs) return;                              // (all CTAs of the cluster alike)
  const Pack pack(p0, a.group);
  const int live = min(kBM, vecs - p0), last_row = pack.row(live - 1);
  const Span keys = part_of(a.mask ? q.cached + q.n : q.cached + last_row + 1, z, a.splits, kFN);

  {
    float4 x[RM * D / 64];                             // all loads in flight
#pragma unroll
    for (int i = 0; i < RM * D / 64; ++i) {
      const int n = threadIdx.x + i * kFThreads, r = n / (D / 4);
      x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < live) x[i] = load4(static_cast<const float*>(a.q) + vec_at<D>(pack, q, h, r, a.q_stride) + n % (D / 4) * 4);
    }
#pragma unroll
    for (int i = 0; i < RM * D / 64; ++i) {
      const int n = threadIdx.x + i * kFThreads;
      *reinterpret_cast<float4*>(&sm.q[n / (D / 4)][n % (D / 4) * 4]) = x[i];
    }
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
  // Tiles travel through registers: the next one is on its way while this one is multiplied.
  constexpr int kPieces = kFN * (D / 4) / kFThreads, kStep = kFThreads / (D / 4);    // float4 a thread, rows between them
  const int my_row = threadIdx.x / (D / 4), my_d = threadIdx.x % (D / 4) * 4;
  float4 kn[kPieces], vn[kPieces];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      kn[i] = vn[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      const int pos = k0 + my_row + i * kStep;
      const long long at = pos < keys.hi ? key_at(a, s, h, pos) : -1;
      if (at >= 0) {
        kn[i] = load4(static_cast<const float*>(a.kv.k) + at + my_d);
        vn[i] = load4(static_cast<const float*>(a.kv.v) + at + my_d);
      }
    }
  };
  fetch(keys.lo);
  // Of the warp's rows (it may have none): all see the keys below `clear`, none sees one from `reach` on.
  const int first = (threadIdx.x >> 5) * 2 * RM;
  const int clear = q.cached + (a.mask ? 0 : pack.row(first) + 1);
  const int reach = first >= live ? 0 : a.mask ? keys.hi : q.cached + pack.row(min(first + 2 * RM, live) - 1) + 1;
  for (int k0 = keys.lo; k0 < keys.hi; k0 += kFN) {
    __syncthreads();                                   // the tile before has been read
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      *reinterpret_cast<float4*>(&sm.k[my_row + i * kStep][my_d]) = kn[i];
      *reinterpret_cast<float4*>(&sm.v[my_row + i * kStep][my_d]) = vn[i];
    }
    __syncthreads();
    if (k0 + kFN < keys.hi) fetch(k0 + kFN);
    if (k0 >= reach) continue;
    float sc[RM][4];
#pragma unroll
    for (int r = 0; r < RM; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c) sc[r][c] = 0.f;
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
          sc[r][c] = fmaf(qq.x, kk[c].x, fmaf(qq.y, kk[c].y, fmaf(qq.z, kk[c].z, fmaf(qq.w, kk[c].w, sc[r][c]))));
      }
    }
    const bool edge = k0 + kFN > clear;                // some key of the tile may be hidden from some row
#pragma unroll
    for (int r = 0; r < RM; ++r) {
      const int row = pack.row(ty * RM + r);
      bool see[4];
      float mx = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        see[c] = !edge || sees(a, q, row, k0 + tx + 16 * c);
        sc[r][c] = see[c] ? sc[r][c] * a.c : -INFINITY;
        mx = fmaxf(mx, sc[r][c]);
      }
#pragma unroll
      for (int w = 8; w; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float mn = fmaxf(m[r], mx), base = mn == -INFINITY ? 0.f : mn, f = exp2f(m[r] - base);
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float p = exp2f(sc[r][c] - base);
        sum += see[c] ? p : 0.f;
        sm.p[ty * RM + r][tx + 16 * c] = see[c] ? p : -0.f;      // (hidden: the sign says so)
      }
      m[r] = mn;
      l[r] = l[r] * f + sum;                           // this thread's share of the row
#pragma unroll
      for (int c = 0; c < kDC; ++c) o[r][c].x *= f, o[r][c].y *= f, o[r][c].z *= f, o[r][c].w *= f;
    }
    __syncwarp();
#pragma unroll 4
    for (int j = 0; j < kFN; j += 4) {                 // (keys behind the end: p = -0)
      float4 p[RM];
#pragma unroll
      for (int r = 0; r < RM; ++r) p[r] = *reinterpret_cast<const float4*>(&sm.p[ty * RM + r][j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float4 vv[kDC];
#pragma unroll
        for (int c = 0; c < kDC; ++c) vv[c] = *reinterpret_cast<const float4*>(&sm.v[j + e][tx * 4 + 64 * c]);
#pragma unroll
        for (int r = 0; r < RM; ++r) {
          const float u = e == 0 ? p[r].x : e == 1 ? p[r].y : e == 2 ? p[r].z : p[r].w;
          if (edge && __float_as_int(u) < 0) continue; // hidden: v may be anything
#pragma unroll
          for (int c = 0; c < kDC; ++c) {
            o[r][c].x = fmaf(u, vv[c].x, o[r][c].x);
            o[r][c].y = fmaf(u, vv[c].y, o[r][c].y);
            o[r][c].z = fmaf(u, vv[c].z, o[r][c].z);
            o[r][c].w = fmaf(u, vv[c].w, o[r][c].w);
          }
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RM; ++r) {
#pragma unroll
    for (int w = 8; w; w >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], w);
  }
  if (a.splits > 1) {
    __syncthreads();                                   // the last tile has been read
    float(&os)[kFN][D + 4] = sm.k;
    static_assert(kBM <= kFN, "o takes the place of the keys");
#pragma unroll
    for (int r = 0; r < RM; ++r) {
#pragma unroll
      for (int c = 0; c < kDC; ++c) *reinterpret_cast<float4*>(&os[ty * RM + r][tx * 4 + 64 * c]) = o[r][c];
      if (tx == 0) sm.m[ty * RM + r] = m[r], sm.l[ty * RM + r] = l[r];
    }
    join_cluster<float, D>(a, q, h, pack, live, &os[0][0], D + 4, sm.m, sm.l);
    return;
  }
#pragma unroll
  for (int r = 0; r < RM; ++r) {
    if (ty * RM + r >= live) continue;
    const float f = normaliser(a, q, pack.row(ty * RM + r), l[r]);
#pragma unroll
    for (int c = 0; c < kDC; ++c)
      store4(static_cast<float*>(a.out) + vec_at<D>(pack, q, h, ty * RM + r, a.out_stride) + tx * 4 + 64 * c,
             make_float4(o[r][c].x * f, o[r][c].y * f, o[r][c].z * f, o[r][c].w * f));
  }
}

// ---- up to 16 packed vectors of a KV head, bf16 ------------------------------------------------------------
// Reading K and V once is all there is to do (4 * 16 flop a byte at most), so the kernel is built for loads: tiles of
// 64 keys by TMA, a box per page and 64 dimensions, two or more tiles in flight per CTA and three CTAs on an SM.
// Warp w multiplies its 16 keys of a tile with the 16 vectors on mma.m16n8k16 (scores: vectors x keys; o: vectors
// x dimensions) and keeps a maximum, a sum and an o of its own, joined at the end.  Probabilities are multiplied as
// a hi + lo pair of bf16 (16 bits): the second product costs nothing next to the loads.
// (With cp.async copies of 16 bytes, 860 instructions a warp and tile, most of them addresses, bound it at half of
// this rate.)
constexpr int kSTile = 64, kSThreads = 128, kSVecs = 16;
template <int D>
struct SLayout {
  static constexpr int kHalf = kSTile * D * 2, kStage = 2 * kHalf;      // K, then V: D / 64 chunks of 64 rows of 128 bytes
  static constexpr int kStages = D == 128 ? 2 : 4;
  static constexpr int kBytes = kStages * kStage + 1024;                // + alignment
  static constexpr int kPitch = D + 4;
  static_assert(4 * kSVecs * kPitch * 4 <= kStages * kStage, "the warps' o takes the stages' place");
};
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
template <int D>
__global__ void __launch_bounds__(kSThreads, 3)
    attn_step_kernel(const AttnArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using L = SLayout<D>;
  constexpr int S = L::kStages, kDC = D / 64, kChunk = kSTile * 128;
  extern __shared__ uint8_t s_smem_raw[];
  __shared__ float sm_m[4][kSVecs], sm_l[4][kSVecs], fin_m[kSVecs], fin_l[kSVecs];
  __shared__ uint64_t full[S];
  __shared__ int abort_flag, n_issued;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(s_smem_raw) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int h = blockIdx.y, split = blockIdx.x;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) mbar_init(&full[i], 1);
    abort_flag = n_issued = 0;
    fence_barrier_init();
    fence_proxy_async();
    asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
  }
  // Loads of a tile: a lane per box (`rows` places of a page) and chunk of 64 dimensions, K and V.
  const int rows = min(a.kv.page_size, kSTile), boxes = kSTile / rows;
  const int my_box = lane / (2 * kDC), my_chunk = lane % kDC;
  const bool my_v = lane / kDC & 1;
  tc::pdl_wait();
  tc::pdl_trigger();
  const int s = a.ranked ? by_tokens(a.ch, blockIdx.z) : blockIdx.z;
  const int32_t* table = a.ch.table + (long long)s * a.ch.table_stride;
  // the first tiles' pages on their way with the lengths (one part only: it starts at key 0)
  const int first_col = (warp * kSTile + my_box * rows) / a.kv.page_size;
  const int first_page = a.splits == 1 && warp < S && my_box < boxes && first_col < a.ch.table_stride ? __ldg(table + first_col) : 0;
  const Seq q = load_seq(a.ch, s);
  if (q.n < 0 && split == 0 && h == 0 && threadIdx.x == 0) report(a.err, MCD_ERR_INVALID_ARG);
  if (q.n <= 0 || q.n > kSVecs / a.group) return;      // (more: the chunk kernel's)
  const int vecs = q.n * a.group;
  const Pack pack(0, a.group);
  const Span keys = part_of(q.cached + q.n, split, a.splits, kSTile);
  const int n_tiles = (keys.hi - keys.lo + kSTile - 1) / kSTile;
  __syncthreads();                                     // the barriers

  // Tile t into its stage, by one warp.
  auto load_tile = [&](int t, bool first) {
    const int pos = keys.lo + t * kSTile + my_box * rows;
    const bool mine = my_box < boxes && pos < keys.hi;
    int page = !mine ? 0 : first && a.splits == 1 ? first_page : __ldg(table + pos / a.kv.page_size);
    if (page < 0 || page >= a.kv.n_pages) {
      report(a.err, MCD_ERR_INVALID_ARG);
      page = 0;
    }
    const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * rows * 128u;
    if (lane == 0) mbar_arrive_expect_tx(&full[t % S], bytes);
    __syncwarp();
    if (mine)
      tma_page(smem + t % S * L::kStage + (my_v ? L::kHalf : 0) + my_chunk * kChunk + my_box * rows * 128, my_v ? &v_map : &k_map,
               my_chunk * 64, pos % a.kv.page_size, h, page, &full[t % S]);
    if (lane == 0) atomicMax(&n_issued, t + 1);
  };
  if (warp < min(S, n_tiles)) load_tile(warp, true);

  // the vectors as A fragments: rows lane / 4 and + 8, columns 2 (lane % 4) and + 8 of every 16
  uint4 qf[D / 16];
  const int r0 = lane >> 2, r1 = r0 + 8;
  {
    auto ptr = [&](int p) { return static_cast<const uint16_t*>(a.q) + vec_at<D>(pack, q, h, p, a.q_stride) + 2 * (lane & 3); };
    const uint16_t *q0 = ptr(min(r0, vecs - 1)), *q1 = ptr(min(r1, vecs - 1));
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      qf[i].x = __ldg(reinterpret_cast<const uint32_t*>(q0 + 16 * i));
      qf[i].y = __ldg(reinterpret_cast<const uint32_t*>(q1 + 16 * i));
      qf[i].z = __ldg(reinterpret_cast<const uint32_t*>(q0 + 16 * i + 8));
      qf[i].w = __ldg(reinterpret_cast<const uint32_t*>(q1 + 16 * i + 8));
    }
  }
  float o[D / 8][4];
#pragma unroll
  for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
  // rows of the vectors (none: nobody reads what such a vector gives)
  const int i0 = r0 < vecs ? pack.row(r0) : -1, i1 = r1 < vecs ? pack.row(r1) : -1;

  bool ok = true;
  for (int t = 0; t < n_tiles; ++t) {
    // (a wait that gave up: what follows is worthless, and reported; the CTA goes on in step and loads no more)
    ok = ok && warp_wait(&full[t % S], t / S & 1, a.err, &abort_flag);
    uint8_t* const v_tile = smem + t % S * L::kStage + L::kHalf;
    const uint32_t vs = smem_u32(v_tile), ks = vs - L::kHalf;
    const int key0 = keys.lo + t * kSTile + 16 * warp;
    if (key0 + 16 > keys.hi) {                         // values behind the keys: zeros
      for (int i = max(0, keys.hi - key0) * 8 + lane; i < 16 * 8; i += 32)
        for (int c = 0; c < kDC; ++c) *reinterpret_cast<uint4*>(v_tile + c * kChunk + 16 * warp * 128 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
      __syncwarp();
    }
    float z[2][4] = {};
    {
      // (16-byte piece c of a row is at c ^ (row % 8))
      const int row = 16 * warp + (lane & 7) + ((lane & 16) >> 1);
      const uint32_t at = ks + row * 128 + ((((lane >> 3) & 1) ^ (row & 7)) << 4);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        uint32_t b[4];
        ldsm4(b, (at ^ (i & 3) << 5) + (i >> 2) * kChunk);
        mma_bf16_16816(z[0], qf[i], b[0], b[1]);
        mma_bf16_16816(z[1], qf[i], b[2], b[3]);
      }
    }
    const bool edge = key0 + 16 > q.cached;
    unsigned hidden = 0;                               // bit 4 n + e: z[n][e] is hidden
    if (edge) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = e < 2 ? i0 : i1;
          if (i >= 0 && !sees(a, q, i, key0 + 8 * n + 2 * (lane & 3) + (e & 1))) hidden |= 1u << (4 * n + e);
        }
    }
    float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        z[n][e] = hidden >> (4 * n + e) & 1 ? -INFINITY : z[n][e] * a.c;
        if (e < 2) x0 = fmaxf(x0, z[n][e]);
        else x1 = fmaxf(x1, z[n][e]);
      }
#pragma unroll
    for (int w = 1; w < 4; w <<= 1) {
      x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, w));
      x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, w));
    }
    const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1);
    const float b0 = n0 == -INFINITY ? 0.f : n0, b1 = n1 == -INFINITY ? 0.f : n1;
    const float f0 = ex2(m0 - b0), f1 = ex2(m1 - b1);
    if (__any_sync(0xffffffffu, n0 != m0 || n1 != m1)) {
#pragma unroll
      for (int i = 0; i < D / 8; ++i) o[i][0] *= f0, o[i][1] *= f0, o[i][2] *= f1, o[i][3] *= f1;
      l0 *= f0, l1 *= f1;
      m0 = n0, m1 = n1;
    }
    uint32_t hi[4], lo[4];                             // A fragment: n = 0: keys 0..7, n = 1: keys 8..15
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const float base = e ? b1 : b0, u = ex2(z[n][e] - base), w = ex2(z[n][e + 1] - base);
        (e ? l1 : l0) += u + w;
        z[n][e] = u, z[n][e + 1] = w;
        const uint32_t x = pack_bf16x2(u, w);
        hi[2 * n + e / 2] = x;
        lo[2 * n + e / 2] = pack_bf16x2(u - bf16_lo_f32(x), w - bf16_hi_f32(x));
      }
    // A product would take an infinity or NaN of a hidden key's value into the row (0 * inf): where one of
    // the tile's new rows has such a value, the sums skip hidden keys one by one.
    bool odd = false;
    if (edge && __any_sync(0xffffffffu, hidden)) {
      const int first = max(q.cached - key0, 0), n = (min(keys.hi - key0, 16) - first) * 8;
      for (int i = lane; i < n; i += 32)
        for (int c = 0; c < kDC; ++c) {
          const uint4 v = *reinterpret_cast<const uint4*>(v_tile + c * kChunk + (16 * warp + first) * 128 + i * 16);
          odd |= !(bf16x2_finite(v.x) && bf16x2_finite(v.y) && bf16x2_finite(v.z) && bf16x2_finite(v.w));
        }
      odd = __any_sync(0xffffffffu, odd);
    }
    if (!odd) {
      const uint4 ph = make_uint4(hi[0], hi[1], hi[2], hi[3]), pl = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      const int row = 16 * warp + (lane & 15);
      const uint32_t at = vs + row * 128 + (((lane >> 4) ^ (row & 7)) << 4);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        uint32_t b[4];
        ldsm4t(b, (at ^ (i & 3) << 5) + (i >> 2) * kChunk);
        mma_bf16_16816(o[2 * i], ph, b[0], b[1]);
        mma_bf16_16816(o[2 * i], pl, b[0], b[1]);
        mma_bf16_16816(o[2 * i + 1], ph, b[2], b[3]);
        mma_bf16_16816(o[2 * i + 1], pl, b[2], b[3]);
      }
    } else {
#pragma unroll 1
      for (int j = 0; j < 16; ++j) {
        const int from = (lane & 28) | (j & 7) >> 1, row = 16 * warp + j;
        float pa = 0.f, pb = 0.f;
        bool ha = false, hb = false;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float u = __shfl_sync(0xffffffffu, z[n][e], from), w = __shfl_sync(0xffffffffu, z[n][e + 2], from);
            const unsigned hd = __shfl_sync(0xffffffffu, hidden, from) >> (4 * n + e);
            if (j == 8 * n + 2 * (from & 3) + e) pa = u, pb = w, ha = hd & 1, hb = hd & 4;
          }
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          const uint32_t v =
              *reinterpret_cast<const uint32_t*>(v_tile + (i >> 3) * kChunk + row * 128 + (((i & 7) ^ (row & 7)) << 4) + 4 * (lane & 3));
          if (!ha) o[i][0] = fmaf(pa, bf16_lo_f32(v), o[i][0]), o[i][1] = fmaf(pa, bf16_hi_f32(v), o[i][1]);
          if (!hb) o[i][2] = fmaf(pb, bf16_lo_f32(v), o[i][2]), o[i][3] = fmaf(pb, bf16_hi_f32(v), o[i][3]);
        }
      }
    }
    __syncthreads();                                   // the tile has been read: its stage takes tile t + S
    if (t + S < n_tiles && warp == (t & 3) && !*(volatile int*)&abort_flag) load_tile(t + S, false);
  }
  __syncthreads();
  if (abort_flag) {                                    // copies that were late land before their place is used again
    if (warp == 0)
      for (int t = max(0, n_issued - S); t < n_issued; ++t) tc::tc_wait(&full[t % S], t / S & 1, a.err, 2000000000ull);
    __syncthreads();
  }
  // the four warps' parts, then their sum over the first one's place
  float* os = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int w = 1; w < 4; w <<= 1) {
    l0 += __shfl_xor_sync(0xffffffffu, l0, w);
    l1 += __shfl_xor_sync(0xffffffffu, l1, w);
  }
  if ((lane & 3) == 0) sm_m[warp][r0] = m0, sm_m[warp][r1] = m1, sm_l[warp][r0] = l0, sm_l[warp][r1] = l1;
#pragma unroll
  for (int i = 0; i < D / 8; ++i) {
    const int d = 8 * i + 2 * (lane & 3);
    if (r0 < vecs) *reinterpret_cast<float2*>(os + (warp * kSVecs + r0) * L::kPitch + d) = make_float2(o[i][0], o[i][1]);
    if (r1 < vecs) *reinterpret_cast<float2*>(os + (warp * kSVecs + r1) * L::kPitch + d) = make_float2(o[i][2], o[i][3]);
  }
  __syncthreads();
  const long long pair = (long long)s * a.kv.n_kv_heads + h;
  for (int t = threadIdx.x; t < vecs * (D / 4); t += kSThreads) {
    const int r = t / (D / 4), d = t % (D / 4) * 4;
    float mx = -INFINITY, sum = 0.f;
    for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sm_m[w][r]);
    const float base = mx == -INFINITY ? 0.f : mx;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = exp2f(sm_m[w][r] - base);
      const float4 y = *reinterpret_cast<const float4*>(os + (w * kSVecs + r) * L::kPitch + d);
      sum = fmaf(f, sm_l[w][r], sum);
      x.x = fmaf(f, y.x, x.x), x.y = fmaf(f, y.y, x.y), x.z = fmaf(f, y.z, x.z), x.w = fmaf(f, y.w, x.w);
    }
    if (a.splits == 1) {
      const float f = normaliser(a, q, pack.row(r), sum);
      store4(static_cast<uint16_t*>(a.out) + vec_at<D>(pack, q, h, r, a.out_stride) + d, make_float4(x.x * f, x.y * f, x.z * f, x.w * f));
    } else if (a.part) {
      float* to = a.part + ((pair * a.splits + split) * kSVecs + r) * (D + 4);
      *reinterpret_cast<float4*>(to + d) = x;
      if (d == 0) to[D] = mx, to[D + 1] = sum;
    } else {
      *reinterpret_cast<float4*>(os + r * L::kPitch + d) = x;       // (this thread alone read these places)
      if (d == 0) fin_m[r] = mx, fin_l[r] = sum;
    }
  }
  if (a.splits > 1 && !a.part) join_cluster<uint16_t, D>(a, q, h, pack, vecs, os, L::kPitch, fin_m, fin_l);
}

// Joins parts in the workspace: a CTA per (KV head, sequence), a thread per four elements of o.
template <int D>
__global__ void __launch_bounds__(256) attn_join_kernel(const AttnArgs a) {
  const int h = blockIdx.x, s = blockIdx.y;
  tc::pdl_wait();
  tc::pdl_trigger();
  const Seq q = load_seq(a.ch, s);
  if (q.n <= 0 || q.n > kSVecs / a.group) return;
  const int vecs = q.n * a.group;
  const Pack pack(0, a.group);
  const long long pair = (long long)s * a.kv.n_kv_heads + h;
  for (int t = threadIdx.x; t < vecs * (D / 4); t += 256) {
    const int r = t / (D / 4), d = t % (D / 4) * 4;
    const float* from = a.part + (pair * a.splits * kSVecs + r) * (D + 4);
    constexpr long long kStep = kSVecs * (D + 4);
    float mx = -INFINITY, sum = 0.f;
#pragma unroll 8
    for (int z = 0; z < a.splits; ++z) mx = fmaxf(mx, __ldcg(from + z * kStep + D));
    const float base = mx == -INFINITY ? 0.f : mx;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int z = 0; z < a.splits; ++z) {
      const float2 ml = __ldcg(reinterpret_cast<const float2*>(from + z * kStep + D));
      const float4 y = __ldcg(reinterpret_cast<const float4*>(from + z * kStep + d));
      const float f = exp2f(ml.x - base);
      sum = fmaf(f, ml.y, sum);
      x.x = fmaf(f, y.x, x.x), x.y = fmaf(f, y.y, x.y), x.z = fmaf(f, y.z, x.z), x.w = fmaf(f, y.w, x.w);
    }
    const float f = normaliser<false>(a, q, pack.row(r), sum);
    store4(static_cast<uint16_t*>(a.out) + vec_at<D>(pack, q, h, r, a.out_stride) + d, make_float4(x.x * f, x.y * f, x.z * f, x.w * f));
  }
}

// Parts of the keys when `work` (tile, KV head) pairs alone would leave SMs idle: enough for `ctas` CTAs per SM,
// each with at least `least` keys, at most `most` parts (a power of two).  The fp32 chunks above
// took 124, 71 or 78 us with 2, 4 or 8 CTAs per SM.
int splits_for(long long work, int max_tokens, int least, int most, int ctas = 2) {
  const int n_sm = sm_count();
  int z = 1;
  while (z < most && work * z < ctas * n_sm && max_tokens / (2 * z) >= least) z *= 2;
  return z;
}

// Whether the order of the sequences matters: CTAs enough that some start when others end.  With it, 128 single rows
// over 17 to 1,023 keys take 50.5 us, without 59.3 (all of 512 keys: 56.0 and 53.7); 24 fp32 chunks 68.8 and 86.0; 128
// fp32 single rows 205 and 255.  It takes a thread per sequence, and the step kernel has kRanked: 129 single rows keep the
// order in which they are given, 59.1.
bool rank(const mcd_chunks& ch, long long ctas) { return ch.n_seqs > 1 && ch.n_seqs <= kRanked && ctas > 2 * sm_count(); }

template <int D, int RM>
cudaError_t launch_f32(AttnArgs a, cudaStream_t st) {
  static std::atomic<unsigned> done{0};
  const int bytes = (int)sizeof(FSmem<D, RM>);
  cudaError_t e = opt_in(attn_f32_kernel<D, RM>, bytes, done);
  if (e != cudaSuccess) return e;
  const long long tiles = ((long long)a.ch.max_rows * a.group + 16 * RM - 1) / (16 * RM);
  a.splits = splits_for(tiles * a.kv.n_kv_heads * a.ch.n_seqs, a.ch.max_tokens, 64, 8, RM == 1 ? 2 : 4);
  a.ranked = rank(a.ch, tiles * a.kv.n_kv_heads * a.ch.n_seqs * a.splits);
  return launch_clusters(attn_f32_kernel<D, RM>, dim3((unsigned)(tiles * a.splits), a.kv.n_kv_heads, a.ch.n_seqs), kFThreads,
                         a.splits, bytes, st, a);
}
template <int D>
cudaError_t launch_f32(const AttnArgs& a, cudaStream_t st) {
  return (long long)a.ch.max_rows * a.group <= 16 ? launch_f32<D, 1>(a, st) : launch_f32<D, 4>(a, st);
}

struct StepPlan {
  int splits;
  bool in_workspace;
};
// Up to 8 parts are joined by the CTAs of a cluster; where that leaves most SMs idle and the
// keys are many, more parts go through the workspace.
StepPlan plan_step(const mcd_paged_kv& kv, const mcd_chunks& ch) {
  const long long pairs = (long long)kv.n_kv_heads * ch.n_seqs;
  const int z = splits_for(pairs, ch.max_tokens, 64, 8);
  const int more = splits_for(pairs, ch.max_tokens, 512, 128);
  return more > 8 ? StepPlan{more, true} : StepPlan{z, false};
}

// Which kernels a bf16 call needs: sequences of up to 16 vectors per KV head go to the step kernel, longer ones to the
// chunk kernel; the bounds tell when there are only the ones or the others.
struct Route {
  bool steps, chunks;
};
// (no sequence has more rows than the buffers)
mcd_chunks bounded(mcd_chunks ch) {
  ch.max_rows = std::min(ch.max_rows, ch.n_rows);
  return ch;
}
Route route_of(const mcd_chunks& ch, int group) {
  const bool chunks = (int64_t)ch.max_rows * group > kSVecs;
  return {!chunks || (int64_t)ch.n_rows < (int64_t)ch.n_seqs * ch.max_rows, chunks};
}

template <int D>
cudaError_t launch_step(AttnArgs a, void* workspace, cudaStream_t st) {
  static std::atomic<unsigned> done{0};
  const int bytes = SLayout<D>::kBytes, rows = std::min(a.kv.page_size, kSTile);
  cudaError_t e = opt_in(attn_step_kernel<D>, bytes, done);
  if (e != cudaSuccess) return e;
  CUtensorMap k_map, v_map;
  if (!page_map(&k_map, a.kv, a.kv.k, a.layer, rows) || !page_map(&v_map, a.kv, a.kv.v, a.layer, rows)) return cudaErrorInvalidValue;
  const StepPlan p = plan_step(a.kv, a.ch);
  a.splits = p.splits;
  a.ranked = rank(a.ch, (long long)a.kv.n_kv_heads * a.ch.n_seqs * p.splits);
  a.part = p.in_workspace ? static_cast<float*>(workspace) : nullptr;
  e = launch_clusters(attn_step_kernel<D>, dim3(a.splits, a.kv.n_kv_heads, a.ch.n_seqs), kSThreads, a.part ? 1 : a.splits, bytes, st, a, k_map,
                      v_map);
  if (e == cudaSuccess && a.part) e = tc::launch(true, attn_join_kernel<D>, dim3(a.kv.n_kv_heads, a.ch.n_seqs), dim3(256), 0, st, a);
  return e;
}

}  // namespace
}  // namespace paged
}  // namespace mcd

using namespace mcd;

extern "C" int64_t mcd_paged_attention_workspace(const mcd_paged_kv* kv, const mcd_chunks* chunks, int32_t n_q_heads) {
  using namespace paged;
  if (check_kv(kv) != MCD_OK || check_chunks(chunks, kv) != MCD_OK || no_rows(chunks) || n_q_heads <= 0) return 0;
  if (kv->dtype != MCD_WEIGHT_BF16 || !route_of(bounded(*chunks), std::max(1, n_q_heads / kv->n_kv_heads)).steps) return 0;
  const StepPlan p = plan_step(*kv, *chunks);
  return p.in_workspace ? 4ll * kv->n_kv_heads * chunks->n_seqs * p.splits * kSVecs * (kv->head_dim + 4) : 0;
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
      !std::isfinite(scale * 1.4426950408889634f))
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
  const AttnArgs a{*kv, bounded(*chunks), q, out, mask, err, q_stride, out_stride, layer, n_q_heads / kv->n_kv_heads, mask_words, 1, 0, nullptr,
                   scale * 1.4426950408889634f, 0};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (kv->dtype == MCD_WEIGHT_F32)
    return cuda_status(kv->head_dim == 64 ? launch_f32<64>(a, st) : launch_f32<128>(a, st));
  AttnArgs b = a;
  cudaError_t e = cudaSuccess;
  const Route r = route_of(a.ch, a.group);
  if (r.steps) e = kv->head_dim == 64 ? launch_step<64>(a, workspace, st) : launch_step<128>(a, workspace, st);
  if (e == cudaSuccess && r.chunks) {
    b.least_vecs = r.steps ? kSVecs : 0;
    e = launch_chunk(b, st);
  }
  return cuda_status(e);
}
