// mcd_paged_attention for more than 16 query vectors of a KV head, bf16: prompts, drafted trees, chunks.
//
// A CTA takes a pair of tiles, 2 x 128 packed query vectors of one (sequence, KV head), against key tiles
// of 128 (mathematics: mcd_attn.cuh).  Everything that multiplies is a 128 x 128 tcgen05 product:
// S = Q K^T (operands in shared memory, S in tensor memory), then O += P V with P read from
// tensor memory, where the softmax threads put it over S.  Roles:
//   warps 0-3 / 4-7   softmax of tile a / b, a thread per row: S from tensor memory, running maximum and sum,
//                     P back.  O is rescaled only when a row's maximum has grown by more than 2^8 (P stays below
//                     256 then, its relative rounding the same): hardly ever after the first tiles.
//   warp 8            copies: K and V tiles by TMA, a box per page and 64 dimensions, through a ring
//   warp 9            issues the products.  While the softmax of one tile runs, the other tile's two products do:
//                     PV_a(j) QK_a(j+1) PV_b(j) QK_b(j+1) ...
//   warp 10           looks at V tiles that some row sees in part: keys past the end become zeros,
//                     and values that are not finite are noted (0 * inf would reach rows that do not see them:
//                     such a pair of tiles is computed again, key by key)
// What bounds it: a pair of tiles has 32 products of 64 cycles a key tile (D = 128; 67 measured, back to back), but
// S to P takes a tile's softmax about 1,700 cycles (exponentials, packing and tensor memory) and its products
// about 1,400, and the other tile fills only part of that.  The product with the first three quarters of P runs under
// the exponentials of the last (halves: 381 us): 3,200 cycles a pair, 1.27 PFLOP/s for 11,559 rows over
// up to 8,500 keys (370 to 382 us; 0.66 of what a library product reaches; tensor pipe 55 % active).
// A CTA fills an SM, and takes about 8 us to start and end (1.5 to its place in the lists, 3 to 4 to the first scores, 2 to
// their P, 1 to 2 to the rows of o written and the next CTA): the pairs with most keys start first (32 x 65 rows over 200 to
// 1,500 keys: 45.4 us, in the sequences' own order 59).
// P is rounded to one bf16, off by 2^-8 of a probability at most, and l sums it unrounded: a hi + lo pair, as the step
// kernel multiplies, would double the second product, half of the tensor work.  Relative to the norm of the result the
// error is 2.2e-3 for those trees and 2.3e-3 for the long prompts; the rounding of the result alone gives 1.7e-3.
// The steps are published ones: running maximum and sum (Milakov and Gimelshein 2018, arXiv 1805.02867), tiles with an
// unnormalised o (Dao et al. 2022, arXiv 2205.14135), the softmax of one tile under the products of another (Shah et al.
// 2024, arXiv 2407.08608).  That o is rescaled only where the maximum has grown far, and that P is handed over in
// parts, are known ideas of recent attention kernels for these tensor cores.
#include <algorithm>

#include "mcd_attn.cuh"

namespace mcd {
namespace paged {
namespace {

constexpr int kCTile = 128;            // keys of a tile, rows of a tile
constexpr int kCRows = 256;            // packed vectors of a CTA
constexpr int kCThreads = 352;
constexpr int kFirst = 6;              // 16-key steps of P's first part: its product runs under the rest of the softmax
constexpr float kGrowth = 8.f;         // log2 of the growth of a maximum that O is rescaled for

template <int D>
struct CLayout {
  static constexpr int kTileBytes = kCTile * D * 2;                     // one Q, K or V tile
  static constexpr int kStages = D == 128 ? 4 : 8;
  static constexpr int kRing = 2 * kTileBytes;
  static constexpr int kBar = kRing + kStages * kTileBytes;             // full[S] empty[S] q s[2] p[2][2] o[2] drain v_full[S / 2] v_seen[S / 2]
  static constexpr int kBars = 3 * kStages + 10;
  static constexpr int kMisc = kBar + kBars * 8;                        // tensor memory address, abort, odd
  static constexpr int kStat = kMisc + 16;                              // m, l of the rows (parts)
  static constexpr int kBytes = kStat + 2 * kCRows * 4 + 1024;          // + alignment
  static constexpr int kPitch = D + 4;
  static_assert(kCRows * kPitch * 4 <= kBar, "the parts of o take the tiles' place");
  static_assert((kRanked + 1) * 8 <= 2 * kCRows * 4, "the order of the sequences takes the statistics' place");
  static_assert(kBytes <= 227 * 1024, "shared memory");
};

// Box of rows of Q: dimensions d .. d + 63 of the heads from h0 on, rows from row0 on.
__device__ __forceinline__ void tma_rows(void* dst, const CUtensorMap* map, int d, int h0, int row0, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          smem_u32(dst)),
      "l"(map), "r"(d), "r"(h0), "r"(row0), "r"(smem_u32(bar))
      : "memory");
}

// B = V: D[m][n] += A[m][k] V[k][n], V in rows of 64 n (128 swizzled bytes), k the row: the n-major layout.  16 k
// are two groups of 8 rows, 1024 bytes apart; the next 64 n are `chunk` bytes on.
__device__ __forceinline__ uint64_t v_desc(uint32_t addr, uint32_t chunk) {
  uint64_t d = 0;
  d |= (uint64_t)((addr >> 4) & 0x3FFFu);
  d |= (uint64_t)((chunk >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= (uint64_t)1u << 46;
  d |= (uint64_t)2u << 61;
  return d;
}
// A from tensor memory.
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}

#define MCD_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define MCD_P8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
#define MCD_I8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of this thread's lane; the values are there after tmem_loaded (which names them).
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
      "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : MCD_R8(r, 0), MCD_R8(r, 8), MCD_R8(r, 16), MCD_R8(r, 24)
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_loaded(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : MCD_P8(r, 0), MCD_P8(r, 8), MCD_P8(r, 16), MCD_P8(r, 24) : : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::MCD_I8(r, 0),
      MCD_I8(r, 8), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// One lane of the warp, the same every time.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p != 0;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Bits of the positions pos0 .. pos0 + 31 that row i sees.
__device__ __forceinline__ uint32_t seen_word(const AttnArgs& a, const Seq& q, int i, int pos0) {
  const int j0 = pos0 - q.cached;                      // new row of bit 0
  auto below = [](int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; };
  if (i >= q.n) return 0u;
  if (!a.mask) return below(i + 1 - j0);
  if (j0 <= -32) return 0xffffffffu;
  const uint32_t* row = a.mask + (long long)(q.row0 + i) * a.mask_words;
  const uint32_t in = below(q.n - j0);
  if (j0 < 0) return (below(-j0) | __ldg(row) << -j0) & in;
  if (!in) return 0u;
  const int w = j0 >> 5;                               // (w < ceil(n / 32) <= mask_words)
  const uint32_t next = w + 1 < a.mask_words ? __ldg(row + w + 1) : 0u;
  return __funnelshift_r(__ldg(row + w), next, j0 & 31) & in;
}

// Packed vector r of the pair over the keys of `keys`, key by key, by a warp; lane d holds dimensions d * D / 32 ...
template <int D>
__device__ __noinline__ void slow_row(const AttnArgs& a, const Seq& q, int s, int h, const Pack& pack, int r, Span keys, float& m, float& l,
                                      float (&o)[D / 32]) {
  constexpr int kE = D / 32;
  const int lane = threadIdx.x & 31, i = pack.row(r);
  const uint16_t* qp = static_cast<const uint16_t*>(a.q) + vec_at<D>(pack, q, h, r, a.q_stride) + lane * kE;
  float x[kE];
  for (int e = 0; e < kE; ++e) x[e] = bf16_bits_to_f32(qp[e]), o[e] = 0.f;
  m = -INFINITY, l = 0.f;
  for (int pos = keys.lo; pos < keys.hi; ++pos) {
    if (!sees(a, q, i, pos)) continue;
    const long long at = key_at(a, s, h, pos);
    if (at < 0) continue;
    const uint16_t* kp = static_cast<const uint16_t*>(a.kv.k) + at + lane * kE;
    const uint16_t* vp = static_cast<const uint16_t*>(a.kv.v) + at + lane * kE;
    float z = 0.f;
    for (int e = 0; e < kE; ++e) z = fmaf(x[e], bf16_bits_to_f32(kp[e]), z);
    for (int w = 16; w; w >>= 1) z += __shfl_xor_sync(0xffffffffu, z, w);
    z *= a.c;
    const float n = fmaxf(m, z), base = n == -INFINITY ? 0.f : n, f = exp2f(m - base), u = exp2f(z - base);
    l = l * f + u;
    for (int e = 0; e < kE; ++e) o[e] = o[e] * f + u * bf16_bits_to_f32(vp[e]);
    m = n;
  }
}

// Pairs of tiles of a sequence (few vectors: the step kernel's).
__device__ __forceinline__ int pairs_of(const AttnArgs& a, const Seq& q) {
  const int vecs = max(q.n, 0) * a.group;
  return vecs <= a.least_vecs ? 0 : (vecs + kCRows - 1) / kCRows;
}

// Sequence of pair `slot` and the pair's number in it (an empty slot: -1, or too large).  The whole block calls it;
// seen: shared memory of kRanked + 1 entries.
__device__ __forceinline__ int2 find_pair(const AttnArgs& a, long long slot, int2* seen) {
  if (a.ranked) {
    // sequences in the order of their tokens, ties in that of their numbers.  Where do i's pairs start?  A warp asks, its
    // lanes hold the others (a thread that went through them all took 55 ns each).
    int2* found = seen + kRanked;
    const int i = threadIdx.x;
    int2 mine = make_int2(0, 0);                       // tokens and pairs
    if (i < a.ch.n_seqs) {
      const Seq q = load_seq(a.ch, i);
      mine = make_int2(q.cached + q.n, pairs_of(a, q));
    }
    if (i < kRanked) seen[i] = mine;                   // (behind the last sequence: no pairs)
    if (i == 0) *found = make_int2(0, -1);
    __syncthreads();
    constexpr int kE = kRanked / 32;
    const int lane = i & 31;
    int2 o[kE];
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] = seen[lane + 32 * e];
#pragma unroll 4
    for (int n = i >> 5; n < a.ch.n_seqs; n += kCThreads / 32) {
      const int2 x = seen[n];
      int at = 0;                                      // (pairs of all: fewer than 2^31, as CTAs)
#pragma unroll
      for (int e = 0; e < kE; ++e) at += o[e].x > x.x || (o[e].x == x.x && lane + 32 * e < n) ? o[e].y : 0;
      at = __reduce_add_sync(0xffffffffu, at);
      if (lane == 0 && at <= slot && slot < at + x.y) *found = make_int2(n, (int)(slot - at));
    }
    __syncthreads();
    return *found;
  }
  // slots of a sequence start at floor(row_start * group / 256) + its number, so that no two overlap; the last slot
  // may be empty
  auto first_slot = [&](int i) { return (long long)__ldg(a.ch.row_start + i) * a.group / kCRows + i; };
  const int s = warp_last_le(a.ch.n_seqs, first_slot, slot);
  return make_int2(s, (int)max(-1ll, min(slot - first_slot(s), 0x7fffffffll)));
}

template <int D>
__global__ void __launch_bounds__(kCThreads, 1)
    attn_chunk_kernel(const AttnArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                      const __grid_constant__ CUtensorMap q_map, const int q_boxes) {
  using L = CLayout<D>;
  constexpr int S = L::kStages, kDC = D / 64;          // 64-dimension chunks of a row
  constexpr uint32_t kChunk = kCTile * 128;            // bytes of one chunk of a tile
  extern __shared__ uint8_t c_smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(c_smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBar);
  uint64_t *empty = full + S, *q_full = empty + S, *s_full = q_full + 1, *p_full = s_full + 2, *o_full = p_full + 4,
           *drain = o_full + 2, *v_full = drain + 1, *v_seen = v_full + S / 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::kMisc + 4);
  volatile int* odd = reinterpret_cast<volatile int*>(smem + L::kMisc + 8);
  float* sm_m = reinterpret_cast<float*>(smem + L::kStat);
  float* sm_l = sm_m + kCRows;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr unsigned long long kWait = 2000000000ull;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    mbar_init(q_full, q_boxes ? 1 : 8);
    mbar_init(drain, 1);
    for (int w = 0; w < 2; ++w) {
      mbar_init(&s_full[w], 1);
      mbar_init(&p_full[2 * w], 4);                    // either part of P
      mbar_init(&p_full[2 * w + 1], 4);
      mbar_init(&o_full[w], 1);
    }
    for (int i = 0; i < S / 2; ++i) {
      mbar_init(&v_full[i], 1);
      mbar_init(&v_seen[i], 1);
    }
    *abort_flag = 0;
    *odd = 0;
    fence_barrier_init();
    fence_proxy_async();
  }
  if (warp == 8 && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // (before the trigger: a kernel that it lets start may take tensor memory, and keep it until this one is done)
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  auto give_back = [&](uint32_t at) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(512u) : "memory");
  };
  tc::pdl_wait();
  tc::pdl_trigger();
  // Which tiles.  The pairs that see most keys come first: CTAs start in the order of their numbers, and a long one that
  // starts last is waited for alone.
  const int part = blockIdx.x % a.splits, h = blockIdx.x / a.splits % a.kv.n_kv_heads;
  const long long slot = blockIdx.x / a.splits / a.kv.n_kv_heads;
  const int2 found = find_pair(a, slot, reinterpret_cast<int2*>(sm_m));
  const int s = __reduce_max_sync(0xffffffffu, found.x), local = __reduce_max_sync(0xffffffffu, found.y);      // (uniform registers)
  const Seq q = load_seq(a.ch, s);
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < a.ch.n_seqs; i += kCThreads)
      if (load_seq(a.ch, i).n < 0) report(a.err, MCD_ERR_INVALID_ARG);
  const int vecs = max(q.n, 0) * a.group, n_pairs = pairs_of(a, q);
  // (all CTAs of a cluster decide alike)
  if (local < 0 || local >= n_pairs) {
    if (warp == 9) give_back(*tmem_slot);
    return;
  }
  const int p0 = (n_pairs - 1 - local) * kCRows;
  const Pack pack(p0, a.group);
  const int i_first = pack.row0, n_vecs = min(kCRows, vecs - p0);
  auto keys_below = [&](int r) {                       // keys that some vector of the pair below r sees
    return a.mask ? q.cached + q.n : q.cached + pack.row(min(r, n_vecs) - 1) + 1;
  };
  const bool two = kCTile < n_vecs;                    // tile b has rows
  const Span keys = part_of(keys_below(kCRows), part, a.splits, kCTile);
  auto tiles_of = [&](int hi) { return max(0, (min(hi, keys.hi) - keys.lo + kCTile - 1) / kCTile); };
  const int n_tiles = tiles_of(keys.hi), n_a = tiles_of(keys_below(kCTile)), n_b = two ? n_tiles : 0;
  // Tiles whose V warp 10 looks at, from this one on: those that end behind the keys or hold a key that some row does
  // not see.  Number n of these has barriers n % (S / 2) of its own (no more V tiles are in the ring): warp 10 waits
  // for every phase of them, as it could not for the ring's, whose earlier phases it has no part in.
  const int first_look = max(0, (min(keys.hi, q.cached + (a.mask ? 0 : i_first + 1)) - keys.lo) / kCTile);

  const uint32_t tmem = *tmem_slot;
  auto s_col = [&](int w) { return tmem + 128u * w; };
  auto o_col = [&](int w) { return tmem + 256u + 128u * w; };
  // load 2 j is K of tile j, 2 j + 1 its V; the barrier that its bytes complete, and the phase
  auto look = [&](uint32_t i) { return i & 1 ? (int)(i >> 1) - first_look : -1; };
  auto load_bar = [&](uint32_t i) { return look(i) < 0 ? &full[i % S] : &v_full[look(i) % (S / 2)]; };
  auto load_phase = [&](uint32_t i) { return look(i) < 0 ? i / S & 1 : (uint32_t)look(i) / (S / 2) & 1; };
  auto stage = [&](uint32_t i) { return smem + L::kRing + i % S * L::kTileBytes; };

  float m = -INFINITY, l = 0.f;                        // softmax threads: of their row
  if (warp == 8) {
    // ---- copies
    const int boxes = kCTile / a.kv.page_size;         // pages of a tile
    const int32_t* table = a.ch.table + (long long)s * a.ch.table_stride;
    const int box = lane / kDC, chunk = lane % kDC;
    uint32_t i = 0;
    if (q_boxes && n_tiles > 0 && lane == 0) {         // Q: a box is the group's heads of kCTile / group rows, packed as it lies
      mbar_arrive_expect_tx(q_full, (two ? 2 : 1) * L::kTileBytes);
      for (int w = 0; w < (two ? 2 : 1); ++w)
        for (int c = 0; c < kDC; ++c)
          tma_rows(smem + w * L::kTileBytes + c * kChunk, &q_map, c * 64, h * a.group, q.row0 + pack.row(w * kCTile), q_full);
    }
    __syncwarp();
    for (int j = 0; j < n_tiles; ++j) {
      const int pos = keys.lo + j * kCTile + box * a.kv.page_size;
      const bool mine = box < boxes && pos < keys.hi;
      int page = mine ? __ldg(table + pos / a.kv.page_size) : 0;
      if (page < 0 || page >= a.kv.n_pages) {
        report(a.err, MCD_ERR_INVALID_ARG);
        page = 0;
      }
      const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * a.kv.page_size * 128u;
      bool go = true;
      for (int kv = 0; kv < 2 && go; ++kv, ++i) {
        if (lane == 0) {
          if (i >= (uint32_t)S) go = tc::tc_wait(&empty[i % S], (i / S - 1) & 1, a.err, kWait);
          if (*abort_flag) go = false;
          if (go) mbar_arrive_expect_tx(load_bar(i), bytes);
          else *abort_flag = 1;
        }
        go = __shfl_sync(0xffffffffu, (int)go, 0);
        if (!go) break;
        if (mine) tma_page(stage(i) + chunk * kChunk + box * a.kv.page_size * 128, kv ? &v_map : &k_map, chunk * 64, 0, h, page, load_bar(i));
      }
      if (!go) break;
    }
    // every copy lands before the CTA may end
    if (lane == 0 && q_boxes && n_tiles > 0) tc::tc_wait(q_full, 0, a.err, kWait);
    if (lane == 0)
      for (uint32_t n = i > (uint32_t)S ? i - S : 0u; n < i; ++n) tc::tc_wait(load_bar(n), load_phase(n), a.err, kWait);
  } else if (warp == 9) {
    // ---- products.  The whole warp runs the loop, so that descriptors stay in uniform registers, and one elected
    // lane (always the same) issues: from a branch of lane 0 alone an issue took 130 cycles, twice what the
    // product does.  One warp for both tiles: with one each, the products of the two mixed and each waited for both
    // (460 against 533 us for 11,559 rows over up to 8,500 keys).
    constexpr uint32_t kQk = tc::idesc_bf16_n(kCTile), kPv = tc::idesc_bf16_n(D) | 1u << 16;       // (bit 16: B is n-major)
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && warp_wait(bar, parity, a.err, abort_flag);
      return ok;
    };
    // (stages, phases and descriptors are counted along: their arithmetic would stand in the products' way)
    const uint64_t q_desc[2] = {tc::sw128_desc(smem_u32(smem)), tc::sw128_desc(smem_u32(smem + L::kTileBytes))};
    const uint64_t k_desc = tc::sw128_desc(smem_u32(smem + L::kRing)), vd0 = v_desc(smem_u32(smem + L::kRing), kChunk);
    constexpr uint32_t kStageStep = L::kTileBytes >> 4;       // (descriptors count 16 bytes)
    auto qk = [&](int w, uint32_t at_k) {
      const uint64_t kd = k_desc + at_k * kStageStep;
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t at = ((k >> 2) * kChunk + (k & 3) * 32) >> 4;
          tc::umma_bf16(s_col(w), q_desc[w] + at, kd + at, kQk, k > 0);
        }
        tc::umma_commit(&s_full[w]);
      }
    };
    auto pv = [&](int w, int j, uint32_t at_v) {
      const uint64_t vd = vd0 + at_v * kStageStep;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (!wait(&p_full[2 * w + half], j & 1)) return;
        tc::tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int k = half ? kFirst : 0; k < (half ? kCTile / 16 : kFirst); ++k)
            umma_ts(o_col(w), s_col(w) + 8 * k, vd + k * (2048 >> 4), kPv, (j | k) != 0);
        }
      }
      if (j + 1 == (w ? n_b : n_a) && elect_one()) tc::umma_commit(&o_full[w]);
    };
    if (n_tiles > 0 && wait(q_full, 0) && wait(&full[0], 0)) {
      tc::tc_fence_after();
      if (n_a > 0) qk(0, 0);
      if (n_b > 0) qk(1, 0);
      uint32_t at_v = 1, phase = 0;                    // K of tile j + 1 is a stage behind V of tile j
      for (int j = 0; j < n_tiles; ++j) {
        const uint32_t at_k = at_v + 1 < S ? at_v + 1 : 0;
        if (j + 1 < n_tiles && !wait(&full[at_k], at_k ? phase : phase ^ 1)) break;
        if (const int n = j - first_look; n < 0) {
          if (!wait(&full[at_v], phase)) break;
        } else if (!wait(&v_full[n % (S / 2)], n / (S / 2) & 1) || !wait(&v_seen[n % (S / 2)], n / (S / 2) & 1)) {
          break;
        }
        if (j < n_a) pv(0, j, at_v);
        if (!ok) break;
        if (j + 1 < n_a) qk(0, at_k);
        if (j < n_b) pv(1, j, at_v);
        if (!ok) break;
        if (j + 1 < n_b) qk(1, at_k);
        if ((at_v += 2) >= S) at_v -= S, phase ^= 1;
      }
    }
    if (elect_one()) tc::umma_commit(drain);
    tc::tc_wait(drain, 0, a.err, kWait);
    __syncwarp();
  } else if (warp == 10) {
    // ---- V tiles that are seen in part
    for (int j = first_look; j < n_tiles; ++j) {
      const uint32_t i = 2 * j + 1;
      if (!warp_wait(load_bar(i), load_phase(i), a.err, abort_flag)) break;
      uint8_t* v = stage(i);
      const int k0 = keys.lo + j * kCTile, first = max(0, q.cached - k0), end = min(kCTile, keys.hi - k0);
      bool bad = false;
#pragma unroll 4
      for (int n = first * 8 + lane; n < end * 8; n += 32)
        for (int c = 0; c < kDC; ++c) {
          const uint4 x = *reinterpret_cast<const uint4*>(v + c * kChunk + n * 16);
          bad |= !(bf16x2_finite(x.x) && bf16x2_finite(x.y) && bf16x2_finite(x.z) && bf16x2_finite(x.w));
        }
      if (bad) *odd = 1;
      for (int n = end * 8 + lane; n < kCTile * 8; n += 32)
        for (int c = 0; c < kDC; ++c) *reinterpret_cast<uint4*>(v + c * kChunk + n * 16) = make_uint4(0u, 0u, 0u, 0u);
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&v_seen[(j - first_look) % (S / 2)]);
    }
  } else {
    // ---- softmax: thread t of tile w has row t
    const int w = warp >> 2, t = threadIdx.x & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    // Q rows into shared memory where no box holds a tile (the group does not divide it), D / 8 lanes a row
    if (!q_boxes) {
      constexpr int kC = D / 8;
      uint4 x[kC];                                     // all in flight
#pragma unroll
      for (int i = 0; i < kC; ++i) {
        const int r = w * kCTile + i * (128 / kC) + t / kC;
        x[i] = make_uint4(0u, 0u, 0u, 0u);
        if (r < n_vecs)
          x[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + vec_at<D>(pack, q, h, r, a.q_stride) + t % kC * 8));
      }
#pragma unroll
      for (int i = 0; i < kC; ++i)
        *reinterpret_cast<uint4*>(smem + w * L::kTileBytes +
                                  tc::sw128_offset(kCTile, i * (128 / kC) + t / kC, t % kC >> 3, t % kC & 7)) = x[i];
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
    }
    const int n_mine = w ? n_b : n_a, mine = w * kCTile + t, row = pack.row(min(mine, n_vecs - 1));
    const int base = w * kCTile + (warp & 3) * 32;     // the warp's first vector
    const bool live = base < n_vecs;
    // keys below this position are seen by every row of the warp
    const int clear = q.cached + (a.mask ? 0 : pack.row(base) + 1);
    float mc = 0.f;                                    // c * (the maximum in use)
    bool ok = true;
    for (int j = 0; j < n_mine; ++j) {
      ok = warp_wait(&s_full[w], j & 1, a.err, abort_flag);
      if (!ok) break;
      // S of the last tile j: every product before it is done, so K of tile j and V of tile j - 1 have been read
      if (w == (n_b > 0) && t == 0) {
        mbar_arrive(&empty[2 * j % S]);
        if (j > 0) mbar_arrive(&empty[(2 * j - 1) % S]);
      }
      tc::tc_fence_after();
      if (live) {
        uint32_t x[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(s_col(w) + lanes + 32 * c, x[c]);
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_loaded(x[c]);
        const int k0 = keys.lo + j * kCTile;
        if (k0 + kCTile > min(clear, keys.hi)) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int pos = k0 + 32 * c, left = keys.hi - pos;
            uint32_t see = seen_word(a, q, row, pos);
            see &= left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
#pragma unroll
            for (int e = 0; e < 32; ++e) x[c][e] = see >> e & 1u ? x[c][e] : 0xff800000u;
          }
        }
        float mx[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          mx[c] = fmaxf(__uint_as_float(x[c][0]), __uint_as_float(x[c][1]));
#pragma unroll
          for (int e = 2; e < 32; e += 2) mx[c] = max3(mx[c], __uint_as_float(x[c][e]), __uint_as_float(x[c][e + 1]));
        }
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        // (m is -inf until the row has seen a key: then any is growth)
        const bool grown = top * a.c > m + kGrowth || (m == -INFINITY && top > -INFINITY);
        if (__any_sync(0xffffffffu, grown)) {
          const float n = fmaxf(m, top * a.c), from = n == -INFINITY ? 0.f : n, f = ex2(m - from);
          if (j > 0) {                                   // (S of tile j came after the product with P of tile j - 1)
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {          // (few columns at a time: S fills the registers)
              uint32_t y[16];
              tc::tmem_ld16_async(o_col(w) + lanes + c, y);
              tc::tmem_wait16(y);
#pragma unroll
              for (int e = 0; e < 16; e += 2) {
                float u, v;
                unpack2(mul2(pack2(__uint_as_float(y[e]), __uint_as_float(y[e + 1])), pack2(f, f)), u, v);
                y[e] = __float_as_uint(u), y[e + 1] = __float_as_uint(v);
              }
              tmem_st16(o_col(w) + lanes + c, y);
            }
          }
          l *= f;
          m = n;
          mc = from;
        }
        const uint64_t scale = pack2(a.c, a.c), shift = pack2(-mc, -mc);
        uint64_t sum[2] = {0ull, 0ull};                // (two zeros each)
        // thirty-two at a time: arguments and exponentials; sums and packing under the next ones' exponentials
        auto exps = [&](int c) {
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            float u, v;
            unpack2(fma2(pack2(__uint_as_float(x[c][e]), __uint_as_float(x[c][e + 1])), scale, shift), u, v);
            x[c][e] = __float_as_uint(u), x[c][e + 1] = __float_as_uint(v);
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) asm volatile("ex2.approx.ftz.f32 %0, %0;" : "+r"(x[c][e]));
        };
        auto take = [&](int c) {
          uint32_t y[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float u = __uint_as_float(x[c][2 * e]), v = __uint_as_float(x[c][2 * e + 1]);
            sum[e & 1] = add2(sum[e & 1], pack2(u, v));
            y[e] = pack_bf16x2(u, v);
          }
          tmem_st16(s_col(w) + lanes + 16 * c, y);
        };
        exps(0);
        exps(1);
        take(0);
        exps(2);
        take(1);
        take(2);
        tmem_stored();                                 // three quarters of P: the product may start
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[2 * w]);
        exps(3);
        take(3);
        float u, v;
        unpack2(add2(sum[0], sum[1]), u, v);
        l += u + v;
        tmem_stored();
      } else if (lane == 0) {
        mbar_arrive(&p_full[2 * w]);
      }
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_full[2 * w + 1]);
    }
    if (ok && n_mine > 0) {
      ok = warp_wait(&o_full[w], 0, a.err, abort_flag);
      tc::tc_fence_after();
    }
    if (a.splits == 1 && ok && live) {
      if (__any_sync(0xffffffffu, *odd)) {
        for (int r = 0; r < 32; ++r) {
          if (base + r >= n_vecs) break;
          float sl, sm, o[D / 32];
          slow_row<D>(a, q, s, h, pack, base + r, keys, sm, sl, o);
          const float f = normaliser(a, q, pack.row(base + r), sl);
          uint16_t* to = static_cast<uint16_t*>(a.out) + vec_at<D>(pack, q, h, base + r, a.out_stride) + lane * (D / 32);
          for (int e = 0; e < D / 32; ++e) to[e] = (uint16_t)pack_bf16x2(o[e] * f, 0.f);
        }
      } else {
        // through the place of the tile's Q (its products are done), so that the lanes write rows and not columns: 1.4 us
        // a CTA otherwise
        const float f = normaliser(a, q, row, l);
        constexpr int kC = D / 8;                      // 16-byte pieces of a row
        uint4* rows = reinterpret_cast<uint4*>(smem + w * L::kTileBytes) + (warp & 3) * 32 * kC;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t y[32];
          tmem_ld32(o_col(w) + lanes + c, y);
          tmem_loaded(y);
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            uint32_t z[4];
#pragma unroll
            for (int g = 0; g < 4; ++g)
              z[g] = pack_bf16x2(__uint_as_float(y[e + 2 * g]) * f, __uint_as_float(y[e + 2 * g + 1]) * f);
            rows[lane * kC + ((c + e) / 8 ^ (lane & 7))] = make_uint4(z[0], z[1], z[2], z[3]);
          }
        }
        __syncwarp();
        uint16_t* out = static_cast<uint16_t*>(a.out);
        const long long at = vec_at<D>(pack, q, h, min(mine, n_vecs - 1), a.out_stride);
#pragma unroll 4
        for (int i = 0; i < kC; ++i) {
          const int r = i * (32 / kC) + lane / kC, piece = lane % kC;
          const long long to = __shfl_sync(0xffffffffu, at, r);
          if (base + r < n_vecs) *reinterpret_cast<uint4*>(out + to + piece * 8) = rows[r * kC + (piece ^ (r & 7))];
        }
      }
    }
  }
  tc::tc_fence_before();
  __syncthreads();                                     // products and copies are done: the tiles' place is free
  tc::tc_fence_after();
  if (a.splits > 1) {
    float* os = reinterpret_cast<float*>(smem);
    if (warp < 8) {
      const int w = warp >> 2, t = threadIdx.x & 127, r = w * kCTile + t, n_mine = w ? n_b : n_a;
      const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
      const int base = w * kCTile + (warp & 3) * 32;
      const bool some = n_mine > 0 && !*abort_flag && base < n_vecs;
      if (some && *odd) {
        for (int n = 0; n < 32 && base + n < n_vecs; ++n) {
          float sm, sl, o[D / 32];
          slow_row<D>(a, q, s, h, pack, base + n, keys, sm, sl, o);
          for (int e = 0; e < D / 32; ++e) os[(base + n) * L::kPitch + lane * (D / 32) + e] = o[e];
          if (lane == 0) sm_m[base + n] = sm, sm_l[base + n] = sl;
        }
      } else {
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t y[32];
          if (some) {
            tmem_ld32(o_col(w) + lanes + c, y);
            tmem_loaded(y);
          }
#pragma unroll
          for (int e = 0; e < 32; e += 4)              // (a row that sees none of the part's keys: P and o are zeros)
            *reinterpret_cast<uint4*>(os + r * L::kPitch + c + e) =
                some ? make_uint4(y[e], y[e + 1], y[e + 2], y[e + 3]) : make_uint4(0u, 0u, 0u, 0u);
        }
        sm_m[r] = some ? m : -INFINITY;
        sm_l[r] = some ? l : 0.f;
      }
    }
    join_cluster<uint16_t, D>(a, q, h, pack, n_vecs, os, L::kPitch, sm_m, sm_l);
    tc::tc_fence_before();
    __syncthreads();
  }
  if (warp == 9) {
    tc::tc_fence_after();
    give_back(tmem);
  }
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
// The driver's encoder, looked up once (null: no driver).
EncodeTiled encoder() {
  static std::atomic<void*> found{nullptr};
  void* fn = found.load(std::memory_order_acquire);
  if (!fn) {
    cudaDriverEntryPointQueryResult got;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &got) != cudaSuccess ||
        got != cudaDriverEntryPointSuccess)
      return nullptr;
    found.store(fn, std::memory_order_release);
  }
  return reinterpret_cast<EncodeTiled>(fn);
}

// Rows of Q, boxes of a tile.
bool rows_map(CUtensorMap* map, const AttnArgs& a) {
  const EncodeTiled encode = encoder();
  if (!encode) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)a.kv.head_dim, (cuuint64_t)a.kv.n_kv_heads * a.group, (cuuint64_t)a.ch.n_rows};
  const cuuint64_t strides[2] = {(cuuint64_t)a.kv.head_dim * 2, (cuuint64_t)a.q_stride * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)a.group, (cuuint32_t)(kCTile / a.group)}, one[3] = {1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.q), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t launch_chunk_d(AttnArgs a, cudaStream_t st) {
  static std::atomic<unsigned> done{0};
  cudaError_t e = opt_in(attn_chunk_kernel<D>, CLayout<D>::kBytes, done);
  if (e != cudaSuccess) return e;
  CUtensorMap k_map, v_map;
  if (!page_map(&k_map, a.kv, a.kv.k, a.layer, a.kv.page_size) ||
      !page_map(&v_map, a.kv, a.kv.v, a.layer, a.kv.page_size)) return cudaErrorInvalidValue;
  // Q by boxes where a tile is whole rows of the group's heads
  CUtensorMap q_map = k_map;
  const int q_boxes = kCTile % a.group == 0;
  if (q_boxes && !rows_map(&q_map, a)) return cudaErrorInvalidValue;
  const long long slots = (long long)a.ch.n_rows * a.group / kCRows + a.ch.n_seqs;
  const long long pairs = std::min(slots, a.ch.n_seqs * (((long long)a.ch.max_rows * a.group + kCRows - 1) / kCRows));
  // one CTA an SM: parts as long as they leave no SM two, each of two tiles at least
  a.splits = 1;
  while (a.splits < 8 && pairs * a.kv.n_kv_heads * a.splits * 2 <= sm_count() && a.ch.max_tokens / (2 * a.splits) >= 2 * kCTile)
    a.splits *= 2;
  // Order costs a CTA 25 ns a sequence, and what it saves is the last CTAs' time: worth it for few of either (65 rows over 200
  // to 1,500 keys each: 32 sequences 45.4 us, without 59; 128, the 1,024 CTAs of 8 heads, 182 and 177).
  a.ranked = a.ch.n_seqs <= kRanked && a.ch.n_seqs * pairs * a.kv.n_kv_heads * a.splits <= 256ll * sm_count();
  // (ordered sequences leave no slots between them)
  const long long grid = (a.ranked ? pairs : slots) * a.kv.n_kv_heads * a.splits;
  if (grid > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  return launch_clusters(attn_chunk_kernel<D>, dim3((unsigned)grid), kCThreads, a.splits, CLayout<D>::kBytes, st, a, k_map, v_map, q_map, q_boxes);
}

}  // namespace

bool page_map(CUtensorMap* map, const mcd_paged_kv& kv, const void* pool, int layer, int rows) {
  const EncodeTiled encode = encoder();
  if (!encode) return false;
  void* base = static_cast<uint8_t*>(const_cast<void*>(pool)) + layer * kv.layer_stride * 2;
  const cuuint64_t dims[4] = {(cuuint64_t)kv.head_dim, (cuuint64_t)kv.page_size, (cuuint64_t)kv.n_kv_heads, (cuuint64_t)kv.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)kv.token_stride * 2, (cuuint64_t)kv.head_stride * 2, (cuuint64_t)kv.page_stride * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1}, one[4] = {1, 1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_chunk(const AttnArgs& a, cudaStream_t st) {
  return a.kv.head_dim == 64 ? launch_chunk_d<64>(a, st) : launch_chunk_d<128>(a, st);
}

}  // namespace paged
}  // namespace mcd
