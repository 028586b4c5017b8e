// Attention of a batch's newest rows over a paged cache whose sequences share
// a prefix (contract: include/lsp.h, work distribution: prefix_sched.cuh).
//
//   s_j = scale q.k_j,  m = max_j s_j,  l = sum_j exp(s_j - m),
//   o = (1/l) sum_j exp(s_j - m) v_j,   lse = m + log l
//
// with the keys cut into segments, each leaving (sum_j 2^(s2_j - m2) v_j, m2,
// l) in base 2, s2 = s log2(e); prefix_join_kernel adds a row's segments with
// weights 2^(m2_seg - max m2).
//
// prefix_attn_fma_kernel: f32 storage, fp32 multiply-adds, 64 rows x 64 keys a
// step, 4 x 4 scores and 4 x (HD / 16) sums a thread.  Where rows fill the tiles (16
// requests of 1 to 16 rows, 32 heads of 128, over 8K: 634 us) it runs at 34 of some 80
// TFLOP/s: 8 shared loads of 16 bytes for 64 multiply-adds keep shared memory's port
// busy 12 cycles of 16, a block of keys has four barriers, and registers and tiles
// leave one CTA of 8 warps on an SM.  Small calls are bound by the latency of their
// rounds of loads (5 over 2K: 18 us).
// bf16 storage: k_prefix_attn_tc.cu.
#include <algorithm>
#include <cstdint>

#include "prefix_sched.cuh"

namespace lsp {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ float ex2a(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

constexpr int kFmaRows = 64, kFmaKeys = 64, kFmaThreads = 256;
// CTAs of an SM: what is on its way in registers (HD / 16 float4) takes too many of them for two where HD = 128
template <int HD>
constexpr int kFmaPerSm = HD == 64 ? 2 : 1;

template <int HD>
struct FmaSmem {
  float q[kFmaRows][HD + 4];
  float kv[kFmaKeys][HD + 4];
  float p[kFmaRows][kFmaKeys + 4];
  int64_t at[2][kFmaKeys];                       // element offset of each key of a block, -1: none
  int64_t line_base[kPrefixMaxSeqs + 1];
  PrefixSeq info[kPrefixMaxSeqs];
  PrefixSched sched;
};

template <int HD>
__device__ void fma_segment(const PrefixAttnParams& p, FmaSmem<HD>& sm, const PrefixSeg& seg) {
  constexpr int kD4 = HD / 4, kCols = HD / 64;   // float4 of a row; float4 output columns of a thread
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int rows = seg.tokens * p.rep, g = seg.head;
  const bool live = 8 * (tid >> 5) < rows;       // the warp has rows (8 of the tile are its)
  const float* q = static_cast<const float*>(p.q);
  __syncthreads();
  for (int i = tid; i < kFmaRows * kD4; i += kFmaThreads) {
    const int r = i / kD4, c = i % kD4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < rows) x = *reinterpret_cast<const float4*>(q + (int64_t)(seg.t0 + r / p.rep) * p.q_stride + (int64_t)(g * p.rep + r % p.rep) * HD + 4 * c);
    *reinterpret_cast<float4*>(&sm.q[r][4 * c]) = x;
  }
  float m[4], l[4], o[4][kCols][4];
  int lim[4];
  const float sl = p.scale * kLog2e;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    m[a] = -INFINITY;
    l[a] = 0.f;
    const int r = 4 * ty + a;
    lim[a] = r >= rows ? 0 : min(seg.see0 + r / p.rep, seg.k_end);
#pragma unroll
    for (int c = 0; c < kCols; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[a][c][e] = 0.f;
  }
  // Keys, then values of a block go through one tile; the next ones are on their
  // way in registers meanwhile.
  float4 ahead[kFmaKeys * kD4 / kFmaThreads];
  auto fetch = [&](const char* pool, int kb) {
#pragma unroll
    for (int i = 0; i < kFmaKeys * kD4 / kFmaThreads; ++i) {
      const int x = tid + i * kFmaThreads;
      const int64_t at = sm.at[kb & 1][x / kD4];
      ahead[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (at >= 0) ahead[i] = *reinterpret_cast<const float4*>(pool + 4 * (at + 4 * (x % kD4)));
    }
  };
  auto store = [&]() {
#pragma unroll
    for (int i = 0; i < kFmaKeys * kD4 / kFmaThreads; ++i) {
      const int x = tid + i * kFmaThreads;
      *reinterpret_cast<float4*>(&sm.kv[x / kD4][4 * (x % kD4)]) = ahead[i];
    }
  };
  auto page_of = [&](int kb) {                   // of this thread's key of block kb; -1: none
    const int pos = seg.k0 + kb * kFmaKeys + tid;
    return tid < kFmaKeys && kb < seg.kb1 && pos < seg.k_end ? seg.tab[pos / p.page] : -1;
  };
  auto put_at = [&](int kb, int pg) {
    if (tid >= kFmaKeys) return;
    const int pos = seg.k0 + kb * kFmaKeys + tid;
    int64_t at = -1;
    if (pg >= 0 && pg < p.pages)
      at = (int64_t)pg * p.s_page + (int64_t)(pos % p.page) * p.s_slot + (int64_t)g * p.s_head;
    else if (kb < seg.kb1 && pos < seg.k_end)
      set_err(p.err, LSP_DEV_BAD_SEQ);
    sm.at[kb & 1][tid] = at;
  };
  put_at(seg.kb0, page_of(seg.kb0));
  __syncthreads();                               // (and q is stored)
  fetch(p.k, seg.kb0);
  for (int kb = seg.kb0; kb < seg.kb1; ++kb) {
    const int key0 = seg.k0 + kb * kFmaKeys;
    const int next = page_of(kb + 1);
    if (kb > seg.kb0) __syncthreads();           // the block before's values are read
    store();
    __syncthreads();
    fetch(p.v, kb);
    if (live) {
      float s[4][4];
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[a][c] = 0.f;
#pragma unroll 2
      for (int d = 0; d < HD; d += 4) {
        float4 x[4], y[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) x[a] = *reinterpret_cast<const float4*>(&sm.q[4 * ty + a][d]);
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = *reinterpret_cast<const float4*>(&sm.kv[tx + 16 * c][d]);
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            s[a][c] = fmaf(x[a].x, y[c].x, s[a][c]);
            s[a][c] = fmaf(x[a].y, y[c].y, s[a][c]);
            s[a][c] = fmaf(x[a].z, y[c].z, s[a][c]);
            s[a][c] = fmaf(x[a].w, y[c].w, s[a][c]);
          }
      }
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        float mx = -INFINITY;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s[a][c] = key0 + tx + 16 * c < lim[a] ? s[a][c] * sl : -INFINITY;
          mx = fmaxf(mx, s[a][c]);
        }
#pragma unroll
        for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
        const float nm = fmaxf(m[a], mx), mb = nm == -INFINITY ? 0.f : nm;
        const float keep = ex2a(m[a] - mb);
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float w = ex2a(s[a][c] - mb);
          sum += w;
          sm.p[4 * ty + a][tx + 16 * c] = w;
        }
#pragma unroll
        for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        l[a] = l[a] * keep + sum;
        m[a] = nm;
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[a][c][e] *= keep;
      }
    }
    __syncthreads();                             // p is stored, k is read
    store();
    if (kb + 1 < seg.kb1) put_at(kb + 1, next);
    __syncthreads();
    if (kb + 1 < seg.kb1) fetch(p.k, kb + 1);
    if (live) {
#pragma unroll 2
      for (int j = 0; j < kFmaKeys; j += 4) {
        float4 w[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) w[a] = *reinterpret_cast<const float4*>(&sm.p[4 * ty + a][j]);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj)
#pragma unroll
          for (int c = 0; c < kCols; ++c) {
            const float4 y = *reinterpret_cast<const float4*>(&sm.kv[j + jj][4 * tx + 64 * c]);
#pragma unroll
            for (int a = 0; a < 4; ++a) {
              const float x = jj == 0 ? w[a].x : jj == 1 ? w[a].y : jj == 2 ? w[a].z : w[a].w;
              o[a][c][0] = fmaf(x, y.x, o[a][c][0]);
              o[a][c][1] = fmaf(x, y.y, o[a][c][1]);
              o[a][c][2] = fmaf(x, y.z, o[a][c][2]);
              o[a][c][3] = fmaf(x, y.w, o[a][c][3]);
            }
          }
      }
    }
  }
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int r = 4 * ty + a;
    if (r >= rows) continue;
    const int64_t at = seg.part + r;
#pragma unroll
    for (int c = 0; c < kCols; ++c)
      *part_chunk<HD>(p.part_o, at, tx + 16 * c) = make_float4(o[a][c][0], o[a][c][1], o[a][c][2], o[a][c][3]);
    if (tx == 0) p.part_ml[at] = make_float2(m[a], l[a]);
  }
}

template <int HD>
__global__ void __launch_bounds__(kFmaThreads, kFmaPerSm<HD>) prefix_attn_fma_kernel(const PrefixAttnParams p) {
  extern __shared__ __align__(16) uint8_t fma_raw[];
  FmaSmem<HD>& sm = *reinterpret_cast<FmaSmem<HD>*>(fma_raw);
  griddep_wait();
  griddep_launch();
  const int cta = blockIdx.x;
  if (threadIdx.x < 32) {
    const PrefixSched s = build_sched<1, kFmaKeys>(p, sm.line_base, sm.info, cta == 0);
    if (threadIdx.x == 0) sm.sched = s;
  }
  __syncthreads();
  PrefixSegs<1, kFmaKeys> segs(p, sm.sched, sm.line_base, sm.info, cta);
  PrefixSeg seg;
  while (segs.next_shared(seg)) fma_segment<HD>(p, sm, seg);
  while (segs.next_own(seg)) fma_segment<HD>(p, sm, seg);
}

// Joins the segments of output rows (token, query head); lane l holds dims
// [l HD/32, (l + 1) HD/32).  The running maxima come first, one segment a lane, so
// that the sums themselves are independent loads.  Where rows are few (they have
// many segments each), four warps take a row's segments in turn.  Where they fill
// the GPU, a warp has up to four heads of one KV head: their segments are found
// once, and their sums lie side by side (16 requests over 32K, a round, when this was
// chosen: 132 us in all with four heads a warp, 139 with one).
//
// Bound by latency: 5 us to find a row's segments in code that is not cached yet,
// and three dependent rounds of loads of some 3 us.  Where the segments are
// follows from the lengths alone, so every CTA finds that out again before it
// waits for the main kernel.  That kernel lets it start only after its own wait, so
// the lengths are final by then; but what a grid reads before it has waited itself
// need not be what the calls before wrote, so the lengths are read once more after
// the wait, and the work is laid out again should they differ.  (16 x 1 row over
// 32K: 45.6 us; 43.7 without reading again, 49.5 with all of it after the wait.)
constexpr int kJoinRows = 4, kJoinHeads = 4, kJoinPerSm = 4;
template <typename T, int HD, int kUnitTiles, int kBlock, int kWarps, int kHeads>
__global__ void __launch_bounds__(32 * kJoinRows * kWarps, kWarps > 1 ? 2 : kJoinPerSm) prefix_join_kernel(const PrefixAttnParams p) {
  static_assert(kWarps == 1 || kHeads == 1, "warps that share a row have one");
  constexpr int kVec = HD / 32, kAhead = kWarps > 1 ? 6 : 2;
  extern __shared__ __align__(16) uint8_t join_raw[];
  __shared__ float s_o[kWarps > 1 ? kJoinRows * kWarps : 1][HD], s_l[kJoinRows * kWarps];
  __shared__ PrefixSched s_sched;
  __shared__ int s_pieces[2];
  PrefixSeq* info = reinterpret_cast<PrefixSeq*>(join_raw);
  int64_t* line_base = reinterpret_cast<int64_t*>(info + p.n);
  int64_t* begin = line_base + p.n + 1;          // [grid + 1]: piece_begin
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp / kJoinRows;
  bool waited = false, again = true;
  while (again) {
    if (warp == 0) {
      const PrefixSched s = build_sched<kUnitTiles, kBlock>(p, line_base, info, false);
      if (lane == 0) s_sched = s;
    }
    __syncthreads();
    const PrefixSched s = s_sched;
    for (int c = threadIdx.x; c <= p.grid; c += blockDim.x) begin[c] = piece_begin(s, c);
    // the most pieces that have part of a shared item of a unit but the last, of the last
    if (threadIdx.x < 2)
      s_pieces[threadIdx.x] = s.whole < s.items ? (int)div_floor((int64_t)(threadIdx.x ? s.len_last : s.len_two) * s.ctas, s.line) + 2 : 1;
    __syncthreads();
    // the last CTA whose piece begins at or before place x of the line: an estimate, and what rounding leaves
    const float per_place = __fdividef((float)s.ctas, (float)s.line);
    auto piece_at = [&](int64_t x) {
      int c = min((int)((float)x * per_place), s.ctas - 1);
      while (c + 1 < s.ctas && begin[c + 1] <= x) ++c;
      while (begin[c] > x) --c;
      return c;
    };
    const int parts = cdiv(p.rep, kHeads), per = cdiv(p.rep, parts);   // of a KV head's query heads, and heads of one
    const int64_t rows = (int64_t)p.total * p.nkv * parts;
    again = false;
    for (int64_t w0 = (int64_t)blockIdx.x * kJoinRows; w0 < rows; w0 += (int64_t)gridDim.x * kJoinRows) {
      const int64_t mine = w0 + warp % kJoinRows;
      const int64_t w = mine < rows ? mine : rows - 1;   // a row past the last does the last's work, and stores nothing
      const int t = (int)div_floor(w, p.nkv * parts), h = (int)(w - (int64_t)t * p.nkv * parts), g = h / parts;
      const int hr = (h - g * parts) * per, heads = min(per, p.rep - hr);
      int lo = -1;                                 // the last sequence that starts at or before t
      for (int i0 = 0; i0 < p.n; i0 += 32)
        lo += __popc(__ballot_sync(0xffffffffu, i0 + lane < p.n && info[i0 + lane].first <= t));
      PrefixSeq r = {-1, 0, 0, 0};
      if (lo >= 0) r = info[lo];
      // segments: of each range of the shared part the (at most `pieces`) CTAs that
      // have part of its item, then those of the own item
      int shared = 0, pieces = 1, own = 0, c0 = 0, u = 0, unit = 0, shared_at = 0, own_at = 0, blocks = 0, cost = 1, shared_cost = 1;
      int64_t first = 0, shared_first = 0;         // places of the own item, and of the first range's
      if (t >= r.first && t < r.first + r.rows) {
        const int tile_rows = p.tok_tile * p.rep;
        if (s.items > 0) {
          const int tile = t / p.tok_tile;
          u = tile / kUnitTiles;
          shared_at = (tile % kUnitTiles) * tile_rows + (t - tile * p.tok_tile) * p.rep + hr;
          const bool last = u + 1 == p.units;
          shared_cost = last ? block_cost<kUnitTiles>(p, p.total - u * kUnitTiles * p.tok_tile) : kCostTwo;
          pieces = s_pieces[last];
          shared = p.splits * pieces;
          shared_first = shared_place(s, g * p.splits, u) - s.whole_line;
        }
        const int i = t - r.first, tile = i / p.tok_tile;
        unit = tile / kUnitTiles;
        own_at = (tile % kUnitTiles) * tile_rows + (i - tile * p.tok_tile) * p.rep + hr;
        first = s.shared_line + line_base[lo];
        for (int u = 0; u < unit; ++u)
          first += (int64_t)item_length<kUnitTiles>(p, r, u, own_blocks<kUnitTiles, kBlock>(p, r, s.base, u)) * p.nkv;
        blocks = own_blocks<kUnitTiles, kBlock>(p, r, s.base, unit);
        cost = block_cost<kUnitTiles>(p, r.rows - unit * kUnitTiles * p.tok_tile);
        const int len = item_length<kUnitTiles>(p, r, unit, blocks);
        first += (int64_t)g * len;
        if (blocks > 0) {
          c0 = piece_at(first);
          own = piece_at(first + len - 1) + 1 - c0;
        }
      }
      const int all = shared + own;
      auto row_of = [&](int q) -> int64_t {        // -1: no such segment
        if (q >= all) return -1;
        const bool sh = q < shared;
        const int range = sh && q >= pieces ? q / pieces : 0, k = sh ? q - range * pieces : q - shared;
        const int item = (g * p.splits + range) * p.units + u, nb = sh ? range_blocks(s, range) : blocks;
        if (sh && item < s.whole) return k == 0 && nb > 0 ? shared_rows<kUnitTiles>(p, s, item, 0) + shared_at : -1;
        const int64_t place = sh ? shared_first + range * s.len_range : first;
        const int c = (sh ? piece_at(place) : c0) + k;
        if (c >= s.ctas) return -1;
        // a CTA may have a piece of the item without any of its blocks
        const int price = sh ? shared_cost : cost;
        if (blocks_before(s, begin[c + 1] - place, nb, price) <= blocks_before(s, begin[c] - place, nb, price)) return -1;
        return sh ? shared_rows<kUnitTiles>(p, s, item, c) + shared_at : own_rows<kUnitTiles>(p, r, unit, g, c) + own_at;
      };
      // the first segment of this lane for the maxima, and for the sums
      int64_t row_m = row_of(lane), row_s = row_m;
      if (kWarps > 1) {
        const int src = lane * kWarps + part;
        row_s = __shfl_sync(0xffffffffu, row_m, src & 31);
        if (src >= 32) row_s = row_of(src);
      }
      if (!waited) {
        griddep_wait();
        griddep_launch();
        waited = true;
        bool changed = false;
        for (int i = threadIdx.x; i < p.n; i += blockDim.x) changed |= !same_seq(p, i, info[i]);
        again = __syncthreads_or(changed);
        if (again) break;
      }
      float m[kHeads], l[kHeads], o[kHeads][kVec];
#pragma unroll
      for (int k = 0; k < kHeads; ++k) m[k] = -INFINITY, l[k] = 0.f;
      for (int q = lane;;) {
        if (row_m >= 0) {
#pragma unroll
          for (int k = 0; k < kHeads; ++k)
            if (k < heads) m[k] = fmaxf(m[k], p.part_ml[row_m + k].x);
        }
        if ((q += 32) >= all) break;
        row_m = row_of(q);
      }
      bool some = false;
#pragma unroll
      for (int k = 0; k < kHeads; ++k) {
        m[k] = warp_max(m[k]);
        some |= m[k] > -INFINITY;
#pragma unroll
        for (int e = 0; e < kVec; ++e) o[k][e] = 0.f;
      }
      for (int q0 = 0; q0 < all && some; q0 += 32 * kWarps) {
        const int64_t row = q0 == 0 ? row_s : row_of(q0 + lane * kWarps + part);
        float x[kHeads];
        bool any = false;
#pragma unroll
        for (int k = 0; k < kHeads; ++k) {
          x[k] = 0.f;
          if (row >= 0 && k < heads) {
            const float2 ml = p.part_ml[row + k];
            x[k] = ml.x == -INFINITY ? 0.f : ex2a(ml.x - m[k]);
            l[k] += x[k] * ml.y;
          }
          any |= x[k] > 0.f;
        }
        for (unsigned left = __ballot_sync(0xffffffffu, any); left;) {
          float y[kAhead][kHeads][kVec], f[kAhead][kHeads];
#pragma unroll
          for (int a = 0; a < kAhead; ++a) {
            const int src = left ? __ffs(left) - 1 : 0;
            const bool on = left != 0;
            left &= left - 1;
            const int64_t at = __shfl_sync(0xffffffffu, row, src);
#pragma unroll
            for (int k = 0; k < kHeads; ++k) {
              f[a][k] = on ? __shfl_sync(0xffffffffu, x[k], src) : 0.f;
#pragma unroll
              for (int e = 0; e < kVec; ++e) y[a][k][e] = 0.f;
              if (f[a][k] > 0.f) {
                if constexpr (kVec == 4) {
                  const float4 z = *part_chunk<HD>(p.part_o, at + k, lane);
                  y[a][k][0] = z.x; y[a][k][1] = z.y; y[a][k][2] = z.z; y[a][k][3] = z.w;
                } else {
                  const float2 z = reinterpret_cast<const float2*>(part_chunk<HD>(p.part_o, at + k, lane >> 1))[lane & 1];
                  y[a][k][0] = z.x; y[a][k][1] = z.y;
                }
              }
            }
          }
#pragma unroll
          for (int a = 0; a < kAhead; ++a)
#pragma unroll
            for (int k = 0; k < kHeads; ++k)
#pragma unroll
              for (int e = 0; e < kVec; ++e) o[k][e] = fmaf(y[a][k][e], f[a][k], o[k][e]);
        }
      }
#pragma unroll
      for (int k = 0; k < kHeads; ++k) l[k] = warp_sum(l[k]);
      if constexpr (kWarps > 1) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) s_o[warp][lane * kVec + e] = o[0][e];
        if (lane == 0) s_l[warp] = l[0];
        __syncthreads();
        if (part == 0) {
          l[0] = 0.f;
          for (int k = 0; k < kWarps; ++k) l[0] += s_l[k * kJoinRows + warp];
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            o[0][e] = 0.f;
            for (int k = 0; k < kWarps; ++k) o[0][e] += s_o[k * kJoinRows + warp][lane * kVec + e];
          }
        }
        __syncthreads();
      }
      if (mine >= rows || part > 0) continue;
#pragma unroll
      for (int k = 0; k < kHeads; ++k) {
        if (k >= heads) break;
        const float inv = l[k] > 0.f ? 1.f / l[k] : 0.f;
        const int64_t to = (int64_t)t * p.nq + g * p.rep + hr + k;
        T* out = static_cast<T*>(p.out) + to * HD + lane * kVec;
        if constexpr (sizeof(T) == 2 && kVec == 4)
          *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(o[k][0] * inv, o[k][1] * inv), pack_bf16(o[k][2] * inv, o[k][3] * inv));
        else
#pragma unroll
          for (int e = 0; e < kVec; ++e) out[e] = from_f<T>(o[k][e] * inv);
        if (p.lse && lane == 0) p.lse[to] = m[k] == -INFINITY ? -INFINITY : (m[k] + log2f(l[k])) * kLn2;
      }
    }
  }
  if (!waited) griddep_wait();
}

template <typename T, int HD, int kUnitTiles, int kBlock>
int launch_join(const PrefixAttnParams& p, cudaStream_t s) {
  const int64_t rows = (int64_t)p.total * p.nq;
  auto ctas = [&](int heads) { return ((int64_t)p.total * p.nkv * ((p.rep + heads - 1) / heads) + kJoinRows - 1) / kJoinRows; };
  const size_t smem = p.n * (sizeof(PrefixSeq) + sizeof(int64_t)) + (p.grid + 2) * sizeof(int64_t);
  // four warps a row while all their CTAs are resident at once, two on an SM (over 8K, 1024 rows: 32.4 us, with
  // one warp for several 33.2; 512 rows 27.6 and 30.5; 2048 rows 53 and 42)
  const bool few = rows <= 2 * kJoinRows * (int64_t)p.num_sms;
  const cudaError_t e =
      few ? launch_pdl(prefix_join_kernel<T, HD, kUnitTiles, kBlock, 4, 1>, dim3((unsigned)ctas(1)), dim3(128 * kJoinRows), smem, s, p)
          : launch_pdl(prefix_join_kernel<T, HD, kUnitTiles, kBlock, 1, kJoinHeads>, dim3((unsigned)std::min<int64_t>(ctas(kJoinHeads), kJoinPerSm * p.num_sms)),
                       dim3(32 * kJoinRows), smem, s, p);
  return e == cudaSuccess ? LSP_OK : LSP_ERR_CUDA;
}

template <int HD>
int launch_fma(const PrefixAttnParams& p, cudaStream_t s) {
  static bool set[8] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return LSP_ERR_CUDA;
  if (dev >= 8 || !set[dev]) {
    if (cudaFuncSetAttribute(prefix_attn_fma_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(FmaSmem<HD>)) !=
        cudaSuccess)
      return LSP_ERR_CUDA;
    if (dev < 8) set[dev] = true;
  }
  if (launch_pdl(prefix_attn_fma_kernel<HD>, dim3(p.grid), dim3(kFmaThreads), sizeof(FmaSmem<HD>), s, p) != cudaSuccess)
    return LSP_ERR_CUDA;
  return launch_join<float, HD, 1, kFmaKeys>(p, s);
}

template <int HD>
int launch_tc(const PrefixAttnParams& p, cudaStream_t s) {
  const int rc = launch_prefix_attn_tc(p, s);
  return rc == LSP_OK ? launch_join<bf16, HD, kPrefixTcTiles, kPrefixTcKeys>(p, s) : rc;
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Key ranges of the shared part.  The line cuts the keys among the CTAs by
// itself, in the fewest segments; ranges only keep the units of a head close to
// each other in the keys: as many as there are CTAs for, if it has several units.
int choose_splits(int heads, int units, int blocks, int grid) {
  return units == 1 ? 1 : std::max(1, std::min(grid / (heads * units), blocks));
}

}  // namespace

size_t prefix_attn_plan(PrefixAttnParams* p, int dtype, int num_sms) {
  const bool tc = dtype == LSP_DTYPE_BF16;
  const int tile = tc ? kPrefixTcRows : kFmaRows, unit_tiles = tc ? kPrefixTcTiles : 1;
  const int block = tc ? kPrefixTcKeys : kFmaKeys, per_sm = tc ? 1 : p->d == 64 ? kFmaPerSm<64> : kFmaPerSm<128>;
  p->tok_tile = tile / p->rep;
  p->units = (p->total + p->tok_tile * unit_tiles - 1) / (p->tok_tile * unit_tiles);
  p->num_sms = num_sms;
  p->grid = std::min(num_sms * per_sm, kPrefixMaxGrid);
  p->splits = choose_splits(p->nkv, p->units, (p->shared_len + block - 1) / block, p->grid);
  // (not of `splits`: the workspace of one shared_len is enough for any)
  const int64_t rows = (int64_t)p->tok_tile * p->rep * unit_tiles, items = std::max<int64_t>((int64_t)p->nkv * p->units, p->grid);
  p->part_rows = (items + 2 * p->grid) * rows + (int64_t)p->nkv * p->rep * p->total;
  p->part_rows = (p->part_rows + 3) / 4 * 4;
  return align256((size_t)p->part_rows * sizeof(float2)) + (size_t)p->part_rows * p->d * sizeof(float);
}

int launch_prefix_attention(PrefixAttnParams p, int dtype, void* ws, cudaStream_t s) {
  char* w = static_cast<char*>(ws);
  p.part_ml = reinterpret_cast<float2*>(w);
  w += align256((size_t)p.part_rows * sizeof(float2));
  p.part_o = reinterpret_cast<float*>(w);
  if (dtype == LSP_DTYPE_BF16) return p.d == 128 ? launch_tc<128>(p, s) : launch_tc<64>(p, s);
  return p.d == 128 ? launch_fma<128>(p, s) : launch_fma<64>(p, s);
}

}  // namespace lsp
