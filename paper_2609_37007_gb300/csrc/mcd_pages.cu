// mcd_pages_fork and mcd_pages_compact (include/mcd_cache.h): the moves of the paged cache's pages.
//
// Fork.  Pages wanted: need(d) = ceil((len + reserve) / page_size); shared are the full(d) = floor(len /
// page_size) filled ones, the rest fresh, but an heir (its parent's first child, with `release`)
// takes over what its parent holds alone.  One CTA (fork_plan_kernel) decides: who is heir, how many fresh
// pages each child wants, their prefix sum, and the first free pages in ascending order, until
// it has as many as are wanted.  Then as many CTAs as there is work write tables and counts and
// copy the part-filled pages' tokens (fork_apply_kernel, a dependent launch).
// Compact.  A gather of tokens; in place each thread moves its 16-byte column of all the
// kept tokens in ascending order, which never overwrites what is still to be read: place i is
// written after keep[i] >= i was read, and keep[j] > keep[i] for what comes later.
//
// Both are bound by HBM (the copied tokens, read and written once) where they copy much, by the
// launches and the plan's chain where they copy little.
#include <algorithm>
#include <climits>

#include "mcd_cache.cuh"

namespace mcd {
namespace paged {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kMaxForkSeqs = 4096;
constexpr int kCopyThreads = 256;

struct ForkArgs {
  mcd_paged_kv kv;
  const int32_t *ref_in, *table_in, *len_in, *parent, *reserve;
  int32_t *ref_out, *table_out, *len_out, *err;
  int32_t* plan;       // workspace: [0] the plan holds, [1] unused, then heir[n_src], first fresh
                       // page of each child [n_dst], the fresh pages [n_dst * dst_cols]
  int n_src, n_dst, src_cols, dst_cols, release;
};
__device__ __forceinline__ int32_t* plan_heir(const ForkArgs& a) { return a.plan + 4; }
__device__ __forceinline__ int32_t* plan_first(const ForkArgs& a) { return a.plan + 4 + a.n_src; }
__device__ __forceinline__ int32_t* plan_fresh(const ForkArgs& a) { return a.plan + 4 + a.n_src + a.n_dst; }

struct Child {
  int parent, len, full, need;
  bool heir;
};
__device__ __forceinline__ Child child_of(const ForkArgs& a, int d, const int32_t* heir) {
  Child c;
  c.parent = __ldg(a.parent + d);
  c.len = c.parent >= 0 ? __ldg(a.len_in + c.parent) : 0;
  const int extra = a.reserve ? __ldg(a.reserve + d) : 0;
  c.full = c.len / a.kv.page_size;
  c.need = (int)(((long long)c.len + extra + a.kv.page_size - 1) / a.kv.page_size);
  c.heir = a.release && c.parent >= 0 && heir[c.parent] == d;
  return c;
}
// Whether an heir takes over its parent's entry c (behind the filled pages).
__device__ __forceinline__ bool taken_over(const ForkArgs& a, int parent, int c) {
  if (c >= a.src_cols) return false;
  const int p = __ldg(a.table_in + (long long)parent * a.src_cols + c);
  return p >= 0 && __ldg(a.ref_in + p) == 1;
}

// Sum of v over the CTA's threads before this one; total: over all.
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int& total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int x = v;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, m);
    if (lane >= m) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  int w = warp_sums[lane];
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, w, m);
    if (lane >= m) w += y;
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  const int before = warp ? __shfl_sync(0xffffffffu, w, warp - 1) : 0;
  __syncthreads();
  return before + x - v;
}

// CTA 0: the plan.  The others: ref_out = ref_in.
__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(const ForkArgs a) {
  __shared__ int heir[kMaxForkSeqs];
  __shared__ int warp_sums[32];
  const int tid = threadIdx.x;
  tc::pdl_wait();
  tc::pdl_trigger();
  if (blockIdx.x > 0) {
    for (long long i = (long long)(blockIdx.x - 1) * kPlanThreads + tid; i < a.kv.n_pages; i += (long long)(gridDim.x - 1) * kPlanThreads)
      a.ref_out[i] = __ldg(a.ref_in + i);
    return;
  }
  for (int s = tid; s < a.n_src; s += kPlanThreads) heir[s] = INT_MAX;
  __syncthreads();
  bool ok = true;
  for (int d = tid; d < a.n_dst; d += kPlanThreads) {
    const int p = __ldg(a.parent + d);
    if (p < -1 || p >= a.n_src) ok = false;
    else if (p >= 0) atomicMin(&heir[p], d);
  }
  for (int s = tid; s < a.n_src; s += kPlanThreads) {
    const int len = __ldg(a.len_in + s);
    if (len < 0 || len > (long long)a.src_cols * a.kv.page_size) ok = false;
  }
  // every entry is a page of the pool or -1, and no -1 stands where the length wants a page
  for (long long i = tid; i < (long long)a.n_src * a.src_cols; i += kPlanThreads) {
    const int p = __ldg(a.table_in + i), s = (int)(i / a.src_cols), c = (int)(i - (long long)s * a.src_cols);
    if (p < -1 || p >= a.kv.n_pages || (p < 0 && (long long)c * a.kv.page_size < __ldg(a.len_in + s))) ok = false;
  }
  ok = __syncthreads_and(ok);
  int want = 0;                                        // fresh pages so far
  if (ok) {
    for (int s = tid; s < a.n_src; s += kPlanThreads) plan_heir(a)[s] = heir[s];
    bool fits = true;
    for (int d0 = 0; d0 < a.n_dst; d0 += kPlanThreads) {
      const int d = d0 + tid;
      int n = 0;
      if (d < a.n_dst) {
        const Child c = child_of(a, d, heir);
        if ((a.reserve && __ldg(a.reserve + d) < 0) || c.need > a.dst_cols) {
          fits = false;
        } else {
          n = c.need - c.full;
          if (c.heir)
            for (int i = c.full; i < c.need; ++i) n -= taken_over(a, c.parent, i);
        }
      }
      int total;
      const int before = block_scan(n, warp_sums, total);
      if (d < a.n_dst) plan_first(a)[d] = want + before;
      want += total;
    }
    ok = __syncthreads_and(fits);
  }
  mcd_status bad = ok ? MCD_OK : MCD_ERR_INVALID_ARG;
  if (ok) {
    int found = 0;
    for (long long p0 = 0; p0 < a.kv.n_pages && found < want; p0 += 4 * kPlanThreads) {
      int pages[4], n = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const long long p = p0 + 4ll * tid + i;
        if (p < a.kv.n_pages && __ldg(a.ref_in + p) == 0) pages[n++] = (int)p;
      }
      int total;
      const int at = found + block_scan(n, warp_sums, total);
      for (int i = 0; i < n && at + i < want; ++i) plan_fresh(a)[at + i] = pages[i];
      found += total;
    }
    if (found < want) bad = MCD_ERR_OOM;
  }
  if (tid == 0) {
    a.plan[0] = bad == MCD_OK;
    if (bad != MCD_OK) report(a.err, bad);
  }
}

// CTAs 0 .. n_dst - 1: row d of the table, its length and counts.  The next n_src: what the old sequences
// give back.  The rest: one (child, layer, k or v) of the part-filled pages' copies each.
__global__ void __launch_bounds__(kCopyThreads) fork_apply_kernel(const ForkArgs a) {
  tc::pdl_wait();
  tc::pdl_trigger();
  if (!__ldcg(a.plan)) return;
  const int32_t* heir = plan_heir(a);
  int b = blockIdx.x;
  if (b < a.n_dst) {
    __shared__ int warp_sums[32];
    const Child c = child_of(a, b, heir);
    int next = plan_first(a)[b];
    if (threadIdx.x == 0) a.len_out[b] = c.len;
    for (int i0 = 0; i0 < a.dst_cols; i0 += kCopyThreads) {
      const int i = i0 + threadIdx.x;
      const bool shared = i < c.full, over = !shared && c.heir && i < c.need && taken_over(a, c.parent, i);
      const bool fresh = i < c.need && !shared && !over;
      // fresh pages before this column: counted over the CTA's columns
      const unsigned m = __ballot_sync(0xffffffffu, fresh);
      const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
      if (lane == 0) warp_sums[warp] = __popc(m);
      __syncthreads();
      int at = next + __popc(m & ((1u << lane) - 1u));
      for (int w = 0; w < kCopyThreads / 32; ++w) {
        if (w < warp) at += warp_sums[w];
        next += warp_sums[w];
      }
      __syncthreads();
      if (i >= a.dst_cols) continue;
      int page = -1;
      if (fresh) page = plan_fresh(a)[at];
      else if (shared || over) page = __ldg(a.table_in + (long long)c.parent * a.src_cols + i);
      a.table_out[(long long)b * a.dst_cols + i] = page;
      // an heir's entries stand for its parent's: their counts stay
      if (page >= 0 && (fresh || !c.heir)) atomicAdd(a.ref_out + page, 1);
    }
    return;
  }
  b -= a.n_dst;
  if (a.release) {
    if (b < a.n_src) {
      const int h = heir[b];
      Child c{};
      if (h < a.n_dst) c = child_of(a, h, heir);       // (no child: INT_MAX)
      for (int i = threadIdx.x; i < a.src_cols; i += kCopyThreads) {
        const int page = __ldg(a.table_in + (long long)b * a.src_cols + i);
        const bool stays = h < a.n_dst && (i < c.full || (i < c.need && taken_over(a, b, i)));
        if (page >= 0 && !stays) atomicSub(a.ref_out + page, 1);
      }
      return;
    }
    b -= a.n_src;
  }
  const int which = b & 1, layer = (b >> 1) % a.kv.n_layers, d = (b >> 1) / a.kv.n_layers;
  const Child c = child_of(a, d, heir);
  const int tokens = c.len % a.kv.page_size;
  if (!tokens || (c.heir && taken_over(a, c.parent, c.full))) return;
  const int es = a.kv.dtype == MCD_WEIGHT_F32 ? 4 : 2, per = a.kv.head_dim * es / 16;       // 16-byte pieces of a token's head
  const long long from = __ldg(a.table_in + (long long)c.parent * a.src_cols + c.full), to = plan_fresh(a)[plan_first(a)[d]];
  const long long base = layer * a.kv.layer_stride;
  uint8_t* pool = static_cast<uint8_t*>(which ? a.kv.v : a.kv.k);
  const uint8_t* src = pool + (base + from * a.kv.page_stride) * es;
  uint8_t* dst = pool + (base + to * a.kv.page_stride) * es;
  // a thread keeps its 16-byte piece and goes through (head, token) in steps of the CTA's other threads, kAhead loads in
  // flight; divisions are outside (in the loop they were most of 126 instructions a piece)
  const int piece = threadIdx.x % per, stride = kCopyThreads / per, dh = stride / tokens, dt = stride % tokens;
  const long long hs = a.kv.head_stride * es, ts = a.kv.token_stride * es;
  int h = threadIdx.x / per / tokens, t = threadIdx.x / per % tokens;
  src += piece * 16;
  dst += piece * 16;
  constexpr int kAhead = 4;
  while (h < a.kv.n_kv_heads) {
    uint4 x[kAhead];
    long long at[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      at[j] = h < a.kv.n_kv_heads ? h * hs + t * ts : -1;
      if (at[j] >= 0) x[j] = __ldcs(reinterpret_cast<const uint4*>(src + at[j]));
      h += dh, t += dt;
      if (t >= tokens) t -= tokens, ++h;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (at[j] >= 0) *reinterpret_cast<uint4*>(dst + at[j]) = x[j];
  }
}

struct CompactArgs {
  mcd_paged_kv kv;
  const int32_t *table_in, *table_out, *start, *keep, *n_keep;
  int32_t *len_out, *err;
  int cols, max_keep;
  int slices;          // in place: (layer, k or v) pairs of a CTA
};

constexpr int kTileTokens = 64;

// Whether two device arrays of int32 share an element (an absent one shares none).
bool overlap(const int32_t* a, int64_t n_a, const int32_t* b, int64_t n_b) {
  const auto x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + 4 * n_b && y < x + 4 * n_a;
}

// Whether sequence s's numbers fit, of its tokens lo .. hi - 1 (every thread of the CTA calls it).
__device__ __forceinline__ bool compact_fits(const CompactArgs& a, int s, int start, int n, bool in_place, int lo, int hi) {
  const long long span = (long long)a.cols * a.kv.page_size;
  bool ok = start >= 0 && n >= 0 && n <= a.max_keep && start + (long long)n <= span;
  if (ok) {
    const int32_t* keep = a.keep + (long long)s * a.max_keep;
    for (int i = lo + threadIdx.x; i < min(hi, n) && ok; i += kCopyThreads) {
      const int k = __ldg(keep + i);
      ok = k >= 0 && start + (long long)k < span && (!in_place || i == 0 || k > __ldg(keep + i - 1));
      if (ok) {
        const int p = __ldg(a.table_in + (long long)s * a.cols + (start + k) / a.kv.page_size);
        const int q = __ldg(a.table_out + (long long)s * a.cols + (start + i) / a.kv.page_size);
        ok = p >= 0 && p < a.kv.n_pages && q >= 0 && q < a.kv.n_pages;
      }
    }
  }
  return __syncthreads_and(ok);
}

// Elements of a layer's pages before head 0 of position `pos`.
__device__ __forceinline__ long long token_at(const CompactArgs& a, const int32_t* table, int s, int pos) {
  return __ldg(table + (long long)s * a.cols + pos / a.kv.page_size) * a.kv.page_stride + pos % a.kv.page_size * a.kv.token_stride;
}

// kInPlace: CTA (0, y, s) moves all tokens of a.slices (layer, k or v) pairs, a thread one column at a time; so many that
// the CTAs just fill the GPU, as each first reads the same numbers (32 sequences, 28 layers, up to 7 tokens: 10.5 us
// with a pair each).  Otherwise CTA (tile, layer and k / v, s) copies its tile of kTileTokens tokens.
template <bool kInPlace>
__global__ void __launch_bounds__(kCopyThreads) compact_kernel(const CompactArgs a) {
  __shared__ long long from[kTileTokens], to[kTileTokens];
  const int s = blockIdx.z;
  tc::pdl_wait();
  tc::pdl_trigger();
  const int start = __ldg(a.start + s), n = __ldg(a.n_keep + s);
  const int first = kInPlace ? 0 : blockIdx.x * kTileTokens;
  const bool lead = blockIdx.x == 0 && blockIdx.y == 0;
  if (!lead && first >= n) return;
  // (in place, and for the length, all of the sequence's numbers; a copy looks at its own)
  const bool all = kInPlace || lead;
  if (!compact_fits(a, s, start, n, kInPlace, all ? 0 : first, all ? INT_MAX : first + kTileTokens)) {
    if (threadIdx.x == 0) report(a.err, MCD_ERR_INVALID_ARG);
    return;
  }
  if (lead && threadIdx.x == 0 && a.len_out) a.len_out[s] = start + n;
  const int es = a.kv.dtype == MCD_WEIGHT_F32 ? 4 : 2, per = a.kv.head_dim * es / 16;
  auto slice = [&](int y) { return static_cast<uint8_t*>(y & 1 ? a.kv.v : a.kv.k) + (y >> 1) * a.kv.layer_stride * es; };
  for (int t0 = first; t0 < (kInPlace ? n : min(n, first + kTileTokens)); t0 += kTileTokens) {
    const int tokens = min(kTileTokens, n - t0);
    for (int i = threadIdx.x; i < tokens; i += kCopyThreads) {
      from[i] = token_at(a, a.table_in, s, start + __ldg(a.keep + (long long)s * a.max_keep + t0 + i)) * es;
      to[i] = token_at(a, a.table_out, s, start + t0 + i) * es;
    }
    __syncthreads();
    if constexpr (kInPlace) {
      const int columns = a.kv.n_kv_heads * per, y0 = blockIdx.y * a.slices, n_y = min(a.slices, 2 * a.kv.n_layers - y0);
      for (int i = threadIdx.x; i < n_y * columns; i += kCopyThreads) {
        const int y = i / columns, c = i - y * columns;
        uint8_t* p = slice(y0 + y) + (c / per) * a.kv.head_stride * es + c % per * 16;
        constexpr int kAhead = 8;
        for (int i0 = 0; i0 < tokens; i0 += kAhead) {  // reads of a batch before its writes
          uint4 x[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
            if (i0 + j < tokens) x[j] = *reinterpret_cast<const uint4*>(p + from[i0 + j]);
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
            if (i0 + j < tokens) *reinterpret_cast<uint4*>(p + to[i0 + j]) = x[j];
        }
      }
    } else {
      // a thread keeps its piece; its tokens one after another, kAhead heads' loads in flight
      const int piece = threadIdx.x % per;
      const long long hs = a.kv.head_stride * es;
      uint8_t* pool = slice(blockIdx.y);
      constexpr int kAhead = 8;
      for (int t = threadIdx.x / per; t < tokens; t += kCopyThreads / per) {
        const uint8_t* src = pool + from[t] + piece * 16;
        uint8_t* dst = pool + to[t] + piece * 16;
        for (int h = 0; h < a.kv.n_kv_heads; h += kAhead, src += kAhead * hs, dst += kAhead * hs) {
          uint4 x[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
            if (h + j < a.kv.n_kv_heads) x[j] = __ldcs(reinterpret_cast<const uint4*>(src + j * hs));
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
            if (h + j < a.kv.n_kv_heads) *reinterpret_cast<uint4*>(dst + j * hs) = x[j];
        }
      }
    }
    __syncthreads();
  }
}

}  // namespace
}  // namespace paged
}  // namespace mcd

using namespace mcd;

extern "C" int64_t mcd_pages_fork_workspace(int32_t n_src, int32_t n_dst, int32_t dst_cols) {
  if (n_src < 0 || n_dst < 0 || dst_cols < 0) return 0;
  return 4ll * (4 + n_src + n_dst + (int64_t)n_dst * dst_cols) + 12;
}

extern "C" mcd_status mcd_pages_fork(const mcd_paged_kv* kv, const int32_t* ref_in, int32_t* ref_out, int32_t n_src,
                                     const int32_t* table_in, int32_t src_cols, const int32_t* len_in, int32_t n_dst,
                                     const int32_t* parent, const int32_t* reserve, int32_t* table_out, int32_t dst_cols,
                                     int32_t* len_out, int32_t release, void* workspace, int64_t workspace_bytes,
                                     int32_t* err, void* stream) {
  using namespace paged;
  const mcd_status s = check_kv(kv);
  if (s != MCD_OK) return s;
  if (!ref_in || !ref_out || ref_in == ref_out || n_src < 0 || n_dst < 0 || src_cols < 0 || dst_cols < 0 || !err)
    return MCD_ERR_INVALID_ARG;
  if (n_src && (!len_in || (src_cols && !table_in))) return MCD_ERR_INVALID_ARG;
  if (n_dst && (!parent || !len_out || (dst_cols && !table_out) || (table_in && table_in == table_out) || (len_in && len_in == len_out)))
    return MCD_ERR_INVALID_ARG;
  if (n_src > kMaxForkSeqs || n_dst > kMaxForkSeqs) return MCD_ERR_UNSUPPORTED;
  const int64_t blocks = (int64_t)n_dst * (1 + 2ll * kv->n_layers) + (release ? n_src : 0);
  if (blocks > INT_MAX || (int64_t)n_dst * dst_cols > INT_MAX) return MCD_ERR_UNSUPPORTED;
  if (!workspace || !aligned16(workspace) || workspace_bytes < mcd_pages_fork_workspace(n_src, n_dst, dst_cols))
    return MCD_ERR_INVALID_ARG;
  const ForkArgs a{*kv, ref_in, table_in, len_in, parent, reserve, ref_out, table_out, len_out, err,
                   static_cast<int32_t*>(workspace), n_src, n_dst, src_cols, dst_cols, release != 0};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int copiers = std::min((kv->n_pages + 4 * kPlanThreads - 1) / (4 * kPlanThreads), 64);
  cudaError_t e = tc::launch(true, fork_plan_kernel, dim3(1 + copiers), dim3(kPlanThreads), 0, st, a);
  if (e == cudaSuccess && blocks) e = tc::launch(true, fork_apply_kernel, dim3((unsigned)blocks), dim3(kCopyThreads), 0, st, a);
  return cuda_status(e);
}

extern "C" mcd_status mcd_pages_compact(const mcd_paged_kv* kv, int32_t n_seqs, const int32_t* table_in,
                                        const int32_t* table_out, int32_t table_cols, const int32_t* start,
                                        const int32_t* keep, int32_t max_keep, const int32_t* n_keep, int32_t* len_out,
                                        int32_t* err, void* stream) {
  using namespace paged;
  const mcd_status s = check_kv(kv);
  if (s != MCD_OK) return s;
  if (n_seqs < 0 || table_cols < 0 || max_keep < 0 || !err) return MCD_ERR_INVALID_ARG;
  if (n_seqs == 0) return MCD_OK;
  if (!start || !n_keep || (table_cols && (!table_in || !table_out)) || (max_keep && !keep)) return MCD_ERR_INVALID_ARG;
  // (a sequence's first CTA writes its length, while others may have yet to read where it starts)
  const int64_t entries = (int64_t)n_seqs * table_cols;
  if (overlap(len_out, n_seqs, start, n_seqs) || overlap(len_out, n_seqs, n_keep, n_seqs) ||
      overlap(len_out, n_seqs, keep, (int64_t)n_seqs * max_keep) || overlap(len_out, n_seqs, table_in, entries) ||
      overlap(len_out, n_seqs, table_out, entries))
    return MCD_ERR_INVALID_ARG;
  if (n_seqs > 65535 || kv->n_layers > 32767 || (int64_t)table_cols * kv->page_size > INT_MAX) return MCD_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool in_place = table_in == table_out;
  // in place: three CTAs an SM, or one for all layers of a sequence
  const int64_t all = 2ll * kv->n_layers * n_seqs, room = 3ll * sm_count();
  const int slices = in_place ? (int)std::min<int64_t>(2 * kv->n_layers, std::max<int64_t>(1, (all + room - 1) / room)) : 1;
  const CompactArgs a{*kv, table_in, table_out, start, keep, n_keep, len_out, err, table_cols, max_keep, slices};
  const dim3 grid(in_place ? 1 : std::max(1, (max_keep + kTileTokens - 1) / kTileTokens), (2 * kv->n_layers + slices - 1) / slices, n_seqs);
  return cuda_status(tc::launch(true, in_place ? compact_kernel<true> : compact_kernel<false>, grid, dim3(kCopyThreads), 0, st, a));
}
