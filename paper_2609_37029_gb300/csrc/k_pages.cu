// Page operators of the target's key/value cache (contracts: include/lsp.h):
// branching, growing, writing, cutting and compacting sequences whose tokens
// lie in fixed-size pages of one pool.
//
// The bookkeeping is exact integer work with one deterministic answer: counts
// of holders only ever change by +-1 per holder (integer atomics commute), and
// pages are handed out by rank -- the k-th page asked for is the k-th lowest
// free one -- so neither depends on the order in which threads run.
//
//   fork, trim   one CTA per pair / entry, one launch
//   write        one warp per row and operand
//   reserve      pages_plan_kernel (one CTA: needs, ranks, table, holders, the
//                list of pages to copy), then pages_copy_kernel
//   compact      pages_compact_plan_kernel (one CTA: ranks, the list of moves),
//                then pages_copy_kernel, which also rewrites the table
//
// branch (fork, reserve 17 tokens, write, trim) of 4 continuations of each of 16
// prompts of 1000-4000 tokens, 32 layers: 76 us for 521 MB copied and written (6.9
// TB/s, the rate of a plain copy).  compact of 2000 live pages of 3000, 8 layers:
// 421 to 432 us for 2.8 GB (6.5 to 6.6 TB/s).  Both are bound by memory; small calls
// by their launches (18 to 21 us from the host, 13 us and 9 us on the device for the
// four calls and for the one).
#include <algorithm>

#include "common.cuh"
#include "lsp_internal.h"

namespace lsp {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kScanBatch = 8;                    // refs per thread and scan step (two int4 loads)
constexpr int kHdrInts = 64;
constexpr int kSmallThreads = 256;
constexpr int kCopyThreads = 256;
constexpr int kCopyBatch = 8;                    // 16-byte loads in flight a lane

// Workspace (ints): header {pages to copy, live pages}; list of source pages,
// of destination pages, filled slots (copies of reserve); the page map.
struct PagesWs {
  int* hdr;
  int* src;
  int* dst;
  int* used;
  int* map;
};

size_t ws_list_ints(int pages) { return (size_t)std::max(pages, kPagesMaxSeqs); }

PagesWs ws_split(void* p, int pages) {
  int* w = static_cast<int*>(p);
  const size_t n = (ws_list_ints(pages) + 3) & ~(size_t)3;
  return {w, w + kHdrInts, w + kHdrInts + n, w + kHdrInts + 2 * n, w + kHdrInts + 3 * n};
}

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// A sequence's length; -1 where the table cannot hold it: an entry with such a sequence is left as it is.
__device__ __forceinline__ int seq_len(const KvCache& c, int s) {
  const int l = c.len[s];
  return l < 0 || l > c.max_pages * c.page ? -1 : l;
}

__device__ __forceinline__ bool in_pool(const KvCache& c, int pg) { return pg >= 0 && pg < c.pages; }

__global__ void __launch_bounds__(kSmallThreads) pages_fork_kernel(const KvCache c, const int* src, const int* dst, int n,
                                                                   unsigned* err) {
  griddep_wait();
  griddep_launch();
  const int i = blockIdx.x, tid = threadIdx.x;
  const int s = src[i], d = dst[i];
  bool bad = s < 0 || s >= c.seqs || d < 0 || d >= c.seqs;
  const int ls = bad ? -1 : seq_len(c, s), ld = bad ? -1 : seq_len(c, d);
  bad = ls < 0 || ld < 0;
  for (int j = tid; j < n; j += kSmallThreads) bad |= src[j] == d || (j < i && dst[j] == d);
  if (__syncthreads_or(bad)) {
    if (tid == 0) set_err(err, LSP_DEV_BAD_SEQ);
    return;
  }
  const int ns = ceil_div(ls, c.page), nd = ceil_div(ld, c.page);
  const int* from = c.table + (size_t)s * c.max_pages;
  int* to = c.table + (size_t)d * c.max_pages;
  bool stray = false;
  for (int k = tid; k < max(ns, nd); k += kSmallThreads)
    stray |= (k < nd && !in_pool(c, to[k])) || (k < ns && !in_pool(c, from[k]));
  if (__syncthreads_or(stray)) {
    if (tid == 0) set_err(err, LSP_DEV_BAD_SEQ);
    return;
  }
  for (int k = tid; k < max(ns, nd); k += kSmallThreads) {
    const int pg = k < ns ? from[k] : -1;
    if (k < nd) atomicSub(c.refs + to[k], 1);
    if (k < ns) atomicAdd(c.refs + pg, 1);
    to[k] = pg;
  }
  if (tid == 0) c.len[d] = ls;                   // (every thread has read it)
}

__global__ void __launch_bounds__(kSmallThreads) pages_trim_kernel(const KvCache c, const int* seqs, const int* new_len,
                                                                   int n, unsigned* err) {
  griddep_wait();
  griddep_launch();
  const int i = blockIdx.x, tid = threadIdx.x;
  const int s = seqs[i], want = new_len[i];
  bool bad = s < 0 || s >= c.seqs || want < 0;
  const int l = bad ? -1 : seq_len(c, s);
  bad = l < 0;
  for (int j = tid; j < i; j += kSmallThreads) bad |= seqs[j] == s;
  if (__syncthreads_or(bad)) {                   // (and every thread has read the length)
    if (tid == 0) set_err(err, LSP_DEV_BAD_SEQ);
    return;
  }
  if (want >= l) return;
  int* row = c.table + (size_t)s * c.max_pages;
  const int end = ceil_div(l, c.page), begin = ceil_div(want, c.page) + tid;
  bool stray = false;
  for (int k = begin; k < end; k += kSmallThreads) stray |= !in_pool(c, row[k]);
  if (__syncthreads_or(stray)) {
    if (tid == 0) set_err(err, LSP_DEV_BAD_SEQ);
    return;
  }
  for (int k = begin; k < end; k += kSmallThreads) {
    atomicSub(c.refs + row[k], 1);
    row[k] = -1;
  }
  if (tid == 0) c.len[s] = want;
}

// Warp w: operand w & 1 (keys, values) of row w >> 1, in 16-byte pieces.
__global__ void __launch_bounds__(kSmallThreads) pages_write_kernel(const KvCache c, const int* seqs, const int* start, int n,
                                                                    const char* k_new, const char* v_new, int64_t row_bytes,
                                                                    int total, int es, unsigned* err) {
  griddep_wait();
  griddep_launch();
  const int lane = threadIdx.x & 31;
  const int w = blockIdx.x * (kSmallThreads / 32) + (threadIdx.x >> 5);
  const int t = w >> 1;                          // (total <= 2^28: w stays below 2^30)
  if (t >= total) return;
  int lo = 0, hi = n;                            // the last entry that starts at or before t
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= t) lo = mid; else hi = mid;
  }
  const int b = start[lo], e = start[lo + 1], s = seqs[lo];
  if (t < b || t >= e) return;                   // a row of no entry
  int pg = -1;
  int pos = -1;
  if (s >= 0 && s < c.seqs && e <= total && b >= 0) {
    const int l = seq_len(c, s);
    pos = l - e + t;
    if (l >= 0 && pos >= 0) pg = c.table[(size_t)s * c.max_pages + pos / c.page];
  }
  if (!in_pool(c, pg)) {
    if (lane == 0) set_err(err, LSP_DEV_BAD_SEQ);
    return;
  }
  const int per_head = c.d * es / 16, vecs = c.nkv * per_head;
  const uint4* from = reinterpret_cast<const uint4*>((w & 1 ? v_new : k_new) + (int64_t)t * row_bytes);
  char* to = (w & 1 ? c.v : c.k) + ((int64_t)pg * c.s_page + (int64_t)(pos % c.page) * c.s_slot) * es;
  for (int i = lane; i < vecs; i += 32)
    reinterpret_cast<uint4*>(to + (int64_t)(i / per_head) * c.s_head * es)[i % per_head] = from[i];
}

// Inclusive sums over the CTA's threads; `all`: the sum of every thread's value.
__device__ __forceinline__ int block_scan(int v, int* s_warp, int* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();                               // the last use of s_warp is over
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  int w = s_warp[lane];                          // kPlanThreads / 32 == 32 warps
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  *all = __shfl_sync(0xffffffffu, w, 31);
  const int before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
  return x + (warp > 0 ? before : 0);
}

// kScanBatch holders' counts from index i on; past the end they read as -1 (neither free nor live).
__device__ __forceinline__ void load_refs(const int* refs, int i, int end, int* r) {
  if (i + kScanBatch <= end && (reinterpret_cast<uintptr_t>(refs + i) & 15) == 0) {
#pragma unroll
    for (int k = 0; k < kScanBatch; k += 4) {
      const int4 x = *reinterpret_cast<const int4*>(refs + i + k);
      r[k] = x.x; r[k + 1] = x.y; r[k + 2] = x.z; r[k + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int k = 0; k < kScanBatch; ++k) r[k] = i + k < end ? refs[i + k] : -1;
  }
}

// One CTA, thread i = entry i.  Bound by latency: some five dependent loads and
// one scan step for every 8192 pages up to the last page that is handed out.
__global__ void __launch_bounds__(kPlanThreads) pages_plan_kernel(const KvCache c, const int* seqs, const int* add, int n,
                                                                  const PagesWs w, unsigned* err) {
  __shared__ int s_warp[32];
  __shared__ int s_seq[kPagesMaxSeqs];
  __shared__ int s_last[kPagesMaxSeqs];          // the shared partly filled page, -1: none
  griddep_wait();
  griddep_launch();
  const int i = threadIdx.x;
  int s = -1, a = 0, l = 0;
  if (i < n) {
    s = seqs[i];
    a = add[i];
    s_seq[i] = s;
  }
  __syncthreads();
  bool ok = i < n && s >= 0 && s < c.seqs && a >= 0;
  for (int j = 0; ok && j < i; ++j) ok = s_seq[j] != s;
  int before = 0, after = 0, last = -1, holders = 0;
  if (ok) {
    l = seq_len(c, s);
    ok = l >= 0 && (int64_t)l + a <= (int64_t)c.max_pages * c.page;
  }
  if (ok) {
    before = ceil_div(l, c.page);
    after = ceil_div(l + a, c.page);
    if (a > 0 && l % c.page) {
      last = c.table[(size_t)s * c.max_pages + before - 1];
      ok = in_pool(c, last);
      if (ok) holders = c.refs[last];
    }
  }
  if (i < n && !ok) set_err(err, LSP_DEV_BAD_SEQ);
  const bool shared = ok && last >= 0 && holders > 1;
  s_last[i] = shared ? last : -1;
  __syncthreads();
  bool copy = false;
  if (shared) {                                  // of r holders, the first r - 1 listed copy
    int earlier = 0;
    for (int j = 0; j < i; ++j) earlier += s_last[j] == last;
    copy = earlier < holders - 1;
  }
  const int need = ok ? after - before + (copy ? 1 : 0) : 0;
  int asked;
  const int upto = block_scan(need, s_warp, &asked);
  // the lowest `asked` free pages, in w.dst by rank
  int found = 0;
  for (int i0 = 0; i0 < c.pages && found < asked; i0 += kPlanThreads * kScanBatch) {
    int r[kScanBatch], z = 0, all;
    const int at = i0 + i * kScanBatch;
    load_refs(c.refs, at, c.pages, r);
#pragma unroll
    for (int k = 0; k < kScanBatch; ++k) z += r[k] == 0;
    int rank = found + block_scan(z, s_warp, &all) - z;
#pragma unroll
    for (int k = 0; k < kScanBatch; ++k)
      if (r[k] == 0) {
        if (rank < asked) w.map[rank] = at + k;
        ++rank;
      }
    found += all;
  }
  __syncthreads();                               // the list is written, every ref is read
  const bool granted = ok && upto <= found;
  if (ok && !granted) set_err(err, LSP_DEV_NO_PAGE);
  const int base = upto - need;
  copy &= granted;
  int copies;
  const int slot = block_scan(copy ? 1 : 0, s_warp, &copies) - 1;
  if (granted) {
    int* row = c.table + (size_t)s * c.max_pages;
    if (copy) {
      const int pg = w.map[base];
      w.src[slot] = last;
      w.dst[slot] = pg;
      w.used[slot] = l % c.page;
      row[before - 1] = pg;
      c.refs[pg] = 1;
      atomicSub(c.refs + last, 1);
    }
    for (int k = copy ? 1 : 0; k < need; ++k) {
      const int pg = w.map[base + k];
      row[before + k - (copy ? 1 : 0)] = pg;
      c.refs[pg] = 1;
    }
    c.len[s] = l + a;
  }
  if (i == 0) w.hdr[0] = copies;
}

// One CTA: count the live pages, rank the holes before that count and the live
// pages behind it, and note for the k-th of each the move between them.
__global__ void __launch_bounds__(kPlanThreads) pages_compact_plan_kernel(const KvCache c, const PagesWs w, int* live_out) {
  __shared__ int s_warp[32];
  griddep_wait();
  griddep_launch();
  const int i = threadIdx.x;
  int mine = 0, live;
  for (int at = i * kScanBatch; at < c.pages; at += kPlanThreads * kScanBatch) {
    int r[kScanBatch];
    load_refs(c.refs, at, c.pages, r);
#pragma unroll
    for (int k = 0; k < kScanBatch; ++k) mine += r[k] > 0;
  }
  block_scan(mine, s_warp, &live);
  int holes = 0, movers = 0;
  for (int i0 = 0; i0 < c.pages; i0 += kPlanThreads * kScanBatch) {
    int r[kScanBatch], z = 0, all;
    const int at = i0 + i * kScanBatch;
    load_refs(c.refs, at, c.pages, r);
    // holes and movers are at most 8192 each here: one scan carries both counts
#pragma unroll
    for (int k = 0; k < kScanBatch; ++k) {
      const bool in = at + k < c.pages, hole = in && at + k < live && r[k] <= 0, mover = in && at + k >= live && r[k] > 0;
      z += (hole ? 1 : 0) + (mover ? 1 << 16 : 0);
    }
    const int upto = block_scan(z, s_warp, &all) - z;
    int hr = holes + (upto & 0xffff), mr = movers + (upto >> 16);
#pragma unroll
    for (int k = 0; k < kScanBatch; ++k) {
      const bool in = at + k < c.pages;
      if (in && at + k < live && r[k] <= 0) w.dst[hr++] = at + k;
      if (in && at + k >= live) {
        if (r[k] > 0)
          w.src[mr++] = at + k;
        else
          w.map[at + k] = at + k;                // a table entry that names a free page stays
      }
    }
    holes += all & 0xffff;
    movers += all >> 16;
  }
  __syncthreads();
  for (int k = i; k < movers; k += kPlanThreads) {
    const int from = w.src[k], to = w.dst[k];
    w.map[from] = to;
    w.used[k] = c.page;
    c.refs[to] = c.refs[from];
    c.refs[from] = 0;
  }
  if (i == 0) {
    w.hdr[0] = movers;
    w.hdr[1] = live;
    if (live_out) *live_out = live;
  }
}

// Copies the listed pages (filled slots only) in every layer, keys and values:
// a unit is one head of one page, a warp takes units in turn.  Sources and
// destinations never meet (new pages are free ones; moves go from behind the
// live count to before it).  remap: also rewrite the table by w.map (compact).
// kQ4: a unit is two runs, the codes of the filled slots and their scales (to the
// next 16 bytes, which are the block's too).
template <bool kQ4>
__global__ void __launch_bounds__(kCopyThreads) pages_copy_kernel(const KvCache c, const PagesWs w, int es, int remap) {
  griddep_wait();
  griddep_launch();
  const int lane = threadIdx.x & 31;
  const int64_t n = w.hdr[0], units = n * c.layers * 2 * c.nkv;
  const int per_slot = kQ4 ? c.d / 32 : c.d * es / 16;   // 16-byte pieces of a slot (its codes): 2, 4, 8, 16 or 32
  const int shift = 31 - __clz(per_slot);
  const int64_t step = (int64_t)gridDim.x * (kCopyThreads / 32);
  for (int64_t u = (int64_t)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); u < units; u += step) {
    const int g = (int)(u % c.nkv);
    int64_t r = u / c.nkv;
    const int kv = (int)(r & 1);
    r >>= 1;
    const int k = (int)(r % n), layer = (int)(r / n);
    char* base = (kv ? c.v : c.k) + ((int64_t)layer * c.s_layer + (int64_t)g * c.s_head) * es;
    const char* from = base + (int64_t)w.src[k] * c.s_page * es;
    char* to = base + (int64_t)w.dst[k] * c.s_page * es;
    const int codes = w.used[k] << shift, vecs = kQ4 ? codes + (w.used[k] * (c.d / 16) + 15) / 16 : codes;
    const int64_t slot_bytes = kQ4 ? per_slot * 16 : c.s_slot * es;
    const int gap = kQ4 ? ((c.page - w.used[k]) << shift) * 16 : 0;     // from the filled slots' codes to the scales
    auto at = [&](int i) { return (i >> shift) * slot_bytes + (i & (per_slot - 1)) * 16 + (kQ4 && i >= codes ? gap : 0); };
    for (int i0 = lane; i0 < vecs; i0 += 32 * kCopyBatch) {
      uint4 x[kCopyBatch];
#pragma unroll
      for (int q = 0; q < kCopyBatch; ++q) {
        const int i = i0 + 32 * q;
        if (i < vecs) x[q] = __ldcs(reinterpret_cast<const uint4*>(from + at(i)));
      }
#pragma unroll
      for (int q = 0; q < kCopyBatch; ++q) {
        const int i = i0 + 32 * q;
        if (i < vecs) __stcs(reinterpret_cast<uint4*>(to + at(i)), x[q]);
      }
    }
  }
  if (!remap || n == 0) return;
  const int live = w.hdr[1];
  const int64_t entries = (int64_t)c.seqs * c.max_pages;
  for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < entries; i += (int64_t)gridDim.x * kCopyThreads) {
    const int pg = c.table[i];
    if (pg >= live && pg < c.pages) c.table[i] = w.map[pg];
  }
}

int status(cudaError_t e) { return e == cudaSuccess ? LSP_OK : LSP_ERR_CUDA; }

// es: bytes of an element, 0 for a cache in 4 bits (its strides are in bytes)
cudaError_t launch_copy(const KvCache& c, const PagesWs& w, int es, int remap, int num_sms, cudaStream_t s) {
  const dim3 grid(num_sms * 8), block(kCopyThreads);
  return es ? launch_pdl(pages_copy_kernel<false>, grid, block, 0, s, c, w, es, remap)
            : launch_pdl(pages_copy_kernel<true>, grid, block, 0, s, c, w, 1, remap);
}

}  // namespace

size_t pages_ws_bytes(int pages) {
  const size_t n = (ws_list_ints(pages) + 3) & ~(size_t)3;
  return (kHdrInts + 4 * n) * sizeof(int);
}

int launch_pages_fork(const KvCache& c, const int* src, const int* dst, int n, unsigned* err, cudaStream_t s) {
  return status(launch_pdl(pages_fork_kernel, dim3(n), dim3(kSmallThreads), 0, s, c, src, dst, n, err));
}

int launch_pages_trim(const KvCache& c, const int* seqs, const int* new_len, int n, unsigned* err, cudaStream_t s) {
  return status(launch_pdl(pages_trim_kernel, dim3(n), dim3(kSmallThreads), 0, s, c, seqs, new_len, n, err));
}

int launch_pages_write(const KvCache& c, const int* seqs, const int* start, int n, const void* k_new, const void* v_new,
                       int64_t row_bytes, int total, int es, unsigned* err, cudaStream_t s) {
  const int per = kSmallThreads / 64;            // rows of a CTA
  return status(launch_pdl(pages_write_kernel, dim3((total + per - 1) / per), dim3(kSmallThreads), 0, s, c, seqs, start, n,
                           static_cast<const char*>(k_new), static_cast<const char*>(v_new), row_bytes, total, es, err));
}

int launch_pages_reserve(const KvCache& c, const int* seqs, const int* add, int n, void* ws, int es, int num_sms,
                         unsigned* err, cudaStream_t s) {
  const PagesWs w = ws_split(ws, c.pages);
  cudaError_t e = launch_pdl(pages_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, c, seqs, add, n, w, err);
  if (e == cudaSuccess)
    e = launch_copy(c, w, es, 0, num_sms, s);
  return status(e);
}

int launch_pages_compact(const KvCache& c, int* live, void* ws, int es, int num_sms, cudaStream_t s) {
  const PagesWs w = ws_split(ws, c.pages);
  cudaError_t e = launch_pdl(pages_compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, c, w, live);
  if (e == cudaSuccess)
    e = launch_copy(c, w, es, 1, num_sms, s);
  return status(e);
}

}  // namespace lsp
