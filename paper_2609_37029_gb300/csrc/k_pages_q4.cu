// Rows into and out of the target's cache (contracts: include/lsp.h): quantising new
// rows into a cache held in 4 bits (format: q4.cuh), and reading any cache back.
//
// Both are bound by memory: a word of codes is eight elements, which a thread has as
// 16 or 32 contiguous bytes of a row, so that a warp moves whole sectors on both
// sides.  Four threads share a group and its scale.
#include <algorithm>

#include "lsp_internal.h"
#include "q4.cuh"

namespace lsp {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;                        // words a lane has in flight

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
  if (t < b || t >= e) return {kNone, 0, 0};
  const int s = seqs[lo];
  if (s < 0 || s >= c.seqs || e > total || b < 0) return {kBad, 0, 0};
  const int l = c.len[s], pos = l - e + t;
  if (l < 0 || l > c.max_pages * c.page || pos < 0) return {kBad, 0, 0};
  const int pg = c.table[(size_t)s * c.max_pages + pos / c.page];
  return {pg >= 0 && pg < c.pages ? kHeld : kStray, pg, pos % c.page};
}

template <typename T>
__device__ __forceinline__ void load8(const char* p, float* x) {
  if constexpr (sizeof(T) == 2) {
    const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = __uint_as_float(w[k] << 16);
      x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
  } else {
    const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
}

// Warp w: operand w & 1 (keys, values) of row w >> 1.
template <typename T>
__global__ void __launch_bounds__(kThreads) pages_write_q4_kernel(const KvCache c, const int* seqs, const int* start, int n,
                                                                  const char* k_new, const char* v_new, int64_t row_bytes,
                                                                  int total, unsigned* err) {
  griddep_wait();
  griddep_launch();
  const int lane = threadIdx.x & 31;
  const int w = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), t = w >> 1;   // (total <= 2^28)
  if (t >= total) return;
  const Row r = find_row(c, seqs, start, n, total, t);
  if (r.kind != kHeld) {
    if (lane == 0 && r.kind != kNone) set_err(err, LSP_DEV_BAD_SEQ);
    return;
  }
  const char* from = (w & 1 ? v_new : k_new) + (int64_t)t * row_bytes;
  char* page = (w & 1 ? c.v : c.k) + (int64_t)r.page * c.s_page;
  const int per_head = c.d / 8, shift = 31 - __clz(per_head), words = c.nkv * per_head;
  const int codes = c.page * (c.d / 2);          // bytes of a block's codes
  for (int i0 = 0; i0 < words; i0 += 32 * kBatch) {
    float x[kBatch][8];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = i0 + 32 * q + lane;
      if (i < words) load8<T>(from + (int64_t)i * 8 * sizeof(T), x[q]);
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = i0 + 32 * q + lane;
      uint32_t a = 0;
      if (i < words) {
#pragma unroll
        for (int e = 0; e < 8; ++e) a = max(a, __float_as_uint(x[q][e]) & 0x7FFFFFFFu);
      }
      a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));    // (a group's four lanes end a row together)
      a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
      if (i >= words) continue;
      const float s = q4_scale(a);
      char* block = page + (int64_t)(i >> shift) * c.s_head;
      const int word = i & (per_head - 1);
      reinterpret_cast<uint32_t*>(block)[r.slot * per_head + word] = q4_codes(x[q], s);
      if ((word & 3) == 0)
        reinterpret_cast<uint16_t*>(block + codes)[r.slot * (per_head >> 2) + (word >> 2)] = (uint16_t)(__float_as_uint(s) >> 16);
    }
  }
}

// Warp w: operand w & 1 of row w >> 1; a piece is a word of codes, or 16 bytes of a cache that holds elements.
template <typename T, bool kQ4>
__global__ void __launch_bounds__(kThreads) pages_read_kernel(const KvCache c, const int* seqs, const int* start, int n,
                                                              char* k_out, char* v_out, int64_t row_bytes, int total,
                                                              unsigned* err) {
  griddep_wait();
  griddep_launch();
  const int lane = threadIdx.x & 31;
  const int w = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), t = w >> 1;
  if (t >= total) return;
  const Row r = find_row(c, seqs, start, n, total, t);
  if (r.kind != kHeld && r.kind != kNone && lane == 0) set_err(err, LSP_DEV_BAD_SEQ);
  if (r.kind == kNone || r.kind == kBad) return;
  char* to = (w & 1 ? v_out : k_out) + (int64_t)t * row_bytes;
  const bool held = r.kind == kHeld;
  constexpr int kElems = kQ4 ? 8 : 16 / (int)sizeof(T);
  const int per_head = c.d / kElems, shift = 31 - __clz(per_head), pieces = c.nkv * per_head;
  const char* page = (w & 1 ? c.v : c.k) + (int64_t)r.page * c.s_page * (kQ4 ? 1 : (int)sizeof(T));
  const int codes = c.page * (c.d / 2);
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
        for (int k = 0; k < 4; ++k) y[k] = held ? q4_pair(x[q].x >> (4 * k), scale) : 0;
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

int status(cudaError_t e) { return e == cudaSuccess ? LSP_OK : LSP_ERR_CUDA; }

dim3 row_grid(int total) { return dim3((unsigned)((total + kThreads / 64 - 1) / (kThreads / 64))); }

}  // namespace

int launch_pages_write_q4(const KvCache& c, const int* seqs, const int* start, int n, const void* k_new, const void* v_new,
                          int64_t row_bytes, int total, int es, unsigned* err, cudaStream_t s) {
  const auto kernel = es == 2 ? pages_write_q4_kernel<bf16> : pages_write_q4_kernel<float>;
  return status(launch_pdl(kernel, row_grid(total), dim3(kThreads), 0, s, c, seqs, start, n, static_cast<const char*>(k_new),
                           static_cast<const char*>(v_new), row_bytes, total, err));
}

int launch_pages_read(const KvCache& c, const int* seqs, const int* start, int n, void* k_out, void* v_out, int64_t row_bytes,
                      int total, int es, bool q4, unsigned* err, cudaStream_t s) {
  const auto kernel = es == 2 ? (q4 ? pages_read_kernel<bf16, true> : pages_read_kernel<bf16, false>)
                              : (q4 ? pages_read_kernel<float, true> : pages_read_kernel<float, false>);
  return status(launch_pdl(kernel, row_grid(total), dim3(kThreads), 0, s, c, seqs, start, n, static_cast<char*>(k_out),
                           static_cast<char*>(v_out), row_bytes, total, err));
}

}  // namespace lsp
