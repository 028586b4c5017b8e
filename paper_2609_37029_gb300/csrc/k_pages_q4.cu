// Rows into and out of the target's cache (contracts: include/lsp.h): quantising new
// rows into a cache held in 4 bits (format: q4.cuh), and reading any cache back.
//
// Both are bound by memory: a word of codes is eight elements, which a thread has as
// 16 or 32 contiguous bytes of a row, so that a warp moves whole sectors on both
// sides.  Four threads share a group and its scale.
//
// Prompts of 1500 to 9000 tokens (41 thousand tokens, 8 heads of 128, bf16): written
// in 42 us (5.1 TB/s: 0.73 of the issue slots, half of the integer pipe), read back in 38
// (5.7 TB/s).  A round's 272 rows take 2 to 3 us each, which is latency: entry, length,
// page, row.
#include <algorithm>

#include "lsp_internal.h"
#include "q4.cuh"

namespace lsp {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;                        // words a lane has in flight

// A value that is the same in all of a warp, as one that the compiler knows to be.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// Row t of a call: the page and slot of its token.  kNone: a row of no entry.
enum RowKind { kNone, kBad, kStray, kHeld };
struct Row {
  RowKind kind;
  int page, slot;
};
__device__ __forceinline__ Row find_row(const KvCache& c, const int* seqs, const int* start, int n, int total, int t) {
  int lo = 0, hi = n;                            // the last entry that starts at or before t
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= t) lo = mid; else hi = mid;
  }
  const int b = start[lo], e = start[lo + 1];
  if (t < b || t >= e || t >= total) return {kNone, 0, 0};
  const int s = seqs[lo];
  if (s < 0 || s >= c.seqs || e > total || b < 0) return {kBad, 0, 0};
  const int l = c.len[s], pos = l - e + t;
  if (l < 0 || l > c.max_pages * c.page || pos < 0) return {kBad, 0, 0};
  const int pg = c.table[(size_t)s * c.max_pages + pos / c.page];
  return {pg >= 0 && pg < c.pages ? kHeld : kStray, pg, pos % c.page};
}

// A CTA's rows, found by a thread each; its warps then take the rows' keys and values in turn.
constexpr int kMostRows = 16;
struct Rows {
  Row row[kMostRows];
};
__device__ __forceinline__ void find_rows(const KvCache& c, const int* seqs, const int* start, int n, int total, int per, Rows& out,
                                          unsigned* err) {
  if ((int)threadIdx.x < per) {
    const Row r = find_row(c, seqs, start, n, total, blockIdx.x * per + threadIdx.x);   // (total <= 2^28)
    if (r.kind == kBad || r.kind == kStray) set_err(err, LSP_DEV_BAD_SEQ);
    out.row[threadIdx.x] = r;
  }
  __syncthreads();
}

template <typename T>
struct Eight {                                   // contiguous elements of a row
  uint4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const char* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 2) {
          x[2 * k] = __uint_as_float(w[k] << 16);
          x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        } else {
          x[4 * i + k] = __uint_as_float(w[k]);
        }
      }
    }
  }
  // the greatest |x|, as the bits of an fp32 number
  __device__ __forceinline__ uint32_t most() const {
    uint32_t a = 0;
    if constexpr (sizeof(T) == 2) {
      // magnitudes of two as 16-bit whole numbers
      const uint32_t w[4] = {v[0].x & 0x7FFF7FFFu, v[0].y & 0x7FFF7FFFu, v[0].z & 0x7FFF7FFFu, v[0].w & 0x7FFF7FFFu};
      a = __vmaxu2(__vmaxu2(w[0], w[1]), __vmaxu2(w[2], w[3]));
      a = max(a & 0xFFFF0000u, a << 16);
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i)
        a = max(max(max(a, v[i].x & 0x7FFFFFFFu), max(v[i].y & 0x7FFFFFFFu, v[i].z & 0x7FFFFFFFu)), v[i].w & 0x7FFFFFFFu);
    }
    return a;
  }
};

// Unit u of a CTA: operand u & 1 (keys, values) of its row u >> 1.  A lane has every 32nd word of the row: always the
// same word of a head, of every (32 / words of a head)-th head.
template <typename T, int HD>
__global__ void __launch_bounds__(kThreads) pages_write_q4_kernel(const KvCache c, const int* seqs, const int* start, int n,
                                                                  const char* k_new, const char* v_new, int64_t row_bytes,
                                                                  int total, int per, unsigned* err) {
  __shared__ Rows rows;
  griddep_wait();
  griddep_launch();
  find_rows(c, seqs, start, n, total, per, rows, err);
  const int lane = threadIdx.x & 31;
  constexpr int kPerHead = HD / 8, kHeads = 32 / kPerHead;       // words of a head, heads of a step
  const int word = lane & (kPerHead - 1), steps = (c.nkv + kHeads - 1) / kHeads;
  for (int u = uniform(threadIdx.x >> 5); u < 2 * per; u += kThreads / 32) {
    Row r = rows.row[u >> 1];
    if (uniform(r.kind) != kHeld) continue;
    r.page = uniform(r.page);
    r.slot = uniform(r.slot);
    const char* from = (u & 1 ? v_new : k_new) + (int64_t)(blockIdx.x * per + (u >> 1)) * row_bytes + lane * 8 * (int)sizeof(T);
    char* block = (u & 1 ? c.v : c.k) + (int64_t)r.page * c.s_page + (int64_t)(lane / kPerHead) * c.s_head;
    const int code_at = (r.slot * kPerHead + word) * 4, scale_at = c.page * (HD / 2) + (r.slot * (kPerHead / 4) + (word >> 2)) * 2;
    for (int i0 = 0; i0 < steps; i0 += kBatch, from += kBatch * 32 * 8 * (int)sizeof(T)) {
      const int left = c.nkv - i0 * kHeads - lane / kPerHead;    // heads from this lane's on
      Eight<T> v[kBatch];
#pragma unroll
      for (int q = 0; q < kBatch; ++q)
        if (q * kHeads < left) v[q].load(from + q * 32 * 8 * (int)sizeof(T));
#pragma unroll
      for (int q = 0; q < kBatch; ++q, block += kHeads * c.s_head) {
        if (i0 + q >= steps) break;
        const bool mine = q * kHeads < left;
        uint32_t a = mine ? v[q].most() : 0;
        a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));  // (a group's four lanes end a row together)
        a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
        if (mine) {
          const float s = q4_scale(a);
          float x[8];
          v[q].get(x);
          *reinterpret_cast<uint32_t*>(block + code_at) = q4_codes<sizeof(T) == 2>(x, s);
          if ((word & 3) == 0) *reinterpret_cast<uint16_t*>(block + scale_at) = (uint16_t)(__float_as_uint(s) >> 16);
        }
        __syncwarp();
      }
    }
  }
}

// The same units; a piece is a word of codes, or 16 bytes of a cache that holds elements.
template <typename T, bool kQ4>
__global__ void __launch_bounds__(kThreads) pages_read_kernel(const KvCache c, const int* seqs, const int* start, int n,
                                                              char* k_out, char* v_out, int64_t row_bytes, int total, int per,
                                                              unsigned* err) {
  __shared__ Rows rows;
  griddep_wait();
  griddep_launch();
  find_rows(c, seqs, start, n, total, per, rows, err);
  const int lane = threadIdx.x & 31;
  const Q4Consts consts;
  constexpr int kElems = kQ4 ? 8 : 16 / (int)sizeof(T);
  const int per_head = c.d / kElems, shift = 31 - __clz(per_head), pieces = c.nkv * per_head;
  const int codes = c.page * (c.d / 2);
  for (int u = threadIdx.x >> 5; u < 2 * per; u += kThreads / 32) {
    const Row r = rows.row[u >> 1];
    if (r.kind == kNone || r.kind == kBad) continue;
    char* to = (u & 1 ? v_out : k_out) + (int64_t)(blockIdx.x * per + (u >> 1)) * row_bytes;
    const bool held = r.kind == kHeld;
    const char* page = (u & 1 ? c.v : c.k) + (int64_t)r.page * c.s_page * (kQ4 ? 1 : (int)sizeof(T));
    for (int i0 = 0; i0 < pieces; i0 += 32 * kBatch) {
      uint4 x[kBatch];
      uint32_t s[kBatch];
#pragma unroll
      for (int q = 0; q < kBatch; ++q) {
        const int i = i0 + 32 * q + lane;
        x[q] = make_uint4(0, 0, 0, 0);
        s[q] = 0;
        if (i >= pieces || !held) continue;
        if constexpr (kQ4) {
          const char* block = page + (int64_t)(i >> shift) * c.s_head;
          const int word = i & (per_head - 1);
          x[q].x = reinterpret_cast<const uint32_t*>(block)[r.slot * per_head + word];
          s[q] = reinterpret_cast<const uint16_t*>(block + codes)[r.slot * (per_head >> 2) + (word >> 2)];
        } else {
          x[q] = reinterpret_cast<const uint4*>(
              page + ((int64_t)r.slot * c.s_slot + (int64_t)(i >> shift) * c.s_head) * (int)sizeof(T))[i & (per_head - 1)];
        }
      }
#pragma unroll
      for (int q = 0; q < kBatch; ++q) {
        const int i = i0 + 32 * q + lane;
        if (i >= pieces) continue;
        uint4* dst = reinterpret_cast<uint4*>(to) + (int64_t)i * (kElems * (int)sizeof(T) / 16);
        if constexpr (!kQ4) {
          __stcs(dst, x[q]);
        } else {
          const uint32_t scale = s[q] | s[q] << 16;
          uint32_t y[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) y[k] = held ? q4_pair(consts, x[q].x >> (4 * k), scale) : 0;
          if constexpr (sizeof(T) == 2) {
            __stcs(dst, make_uint4(y[0], y[1], y[2], y[3]));
          } else {
            __stcs(dst, make_uint4(y[0] << 16, y[0] & 0xFFFF0000u, y[1] << 16, y[1] & 0xFFFF0000u));
            __stcs(dst + 1, make_uint4(y[2] << 16, y[2] & 0xFFFF0000u, y[3] << 16, y[3] & 0xFFFF0000u));
          }
        }
      }
    }
  }
}

int status(cudaError_t e) { return e == cudaSuccess ? LSP_OK : LSP_ERR_CUDA; }

// Rows of a CTA: a warp for each row's keys and values while that leaves no more CTAs than some waves of the GPU.
int rows_per_cta(int total) { return total <= 8192 ? kThreads / 64 : kMostRows; }
dim3 row_grid(int total) { return dim3((unsigned)((total + rows_per_cta(total) - 1) / rows_per_cta(total))); }

}  // namespace

int launch_pages_write_q4(const KvCache& c, const int* seqs, const int* start, int n, const void* k_new, const void* v_new,
                          int64_t row_bytes, int total, int es, unsigned* err, cudaStream_t s) {
  const auto kernel = es == 2 ? (c.d == 128 ? pages_write_q4_kernel<bf16, 128> : pages_write_q4_kernel<bf16, 64>)
                              : (c.d == 128 ? pages_write_q4_kernel<float, 128> : pages_write_q4_kernel<float, 64>);
  return status(launch_pdl(kernel, row_grid(total), dim3(kThreads), 0, s, c, seqs, start, n, static_cast<const char*>(k_new),
                           static_cast<const char*>(v_new), row_bytes, total, rows_per_cta(total), err));
}

int launch_pages_read(const KvCache& c, const int* seqs, const int* start, int n, void* k_out, void* v_out, int64_t row_bytes,
                      int total, int es, bool q4, unsigned* err, cudaStream_t s) {
  const auto kernel = es == 2 ? (q4 ? pages_read_kernel<bf16, true> : pages_read_kernel<bf16, false>)
                              : (q4 ? pages_read_kernel<float, true> : pages_read_kernel<float, false>);
  return status(launch_pdl(kernel, row_grid(total), dim3(kThreads), 0, s, c, seqs, start, n, static_cast<char*>(k_out),
                           static_cast<char*>(v_out), row_bytes, total, rows_per_cta(total), err));
}

}  // namespace lsp
