// Log probabilities of given tokens, entropies and the likeliest alternatives of
// rows of logits (contract: include/lsp.h).
//
// With t_v = (z_v - m) log2(e) / T and e_v = 2^t_v, m the row's largest logit:
//   S = sum e_v,  A = sum e_v t_v
//   logprob = (z_token - m) / T - ln S,  entropy = ln 2 (log2 S - A / S)
// One pass: every thread keeps (m, S, A) of its elements and moves them to a higher
// m as 2^t times (S, A + S t).
//
// The k largest, from the same pass: a thread has a stripe of the CTA's part (every
// 128th piece of 64 bytes), of which it knows at the end the piece with the largest
// logit (the first of several), and the largest of the others.  Each of the k largest
// elements is in one of the k stripes whose first are the largest -- an element in any
// other stripe has k elements before it -- so of those stripes the piece with the
// largest is read again, and the whole stripe where another piece reaches the k-th
// stripe's first too (a few of a hundred).  What is above that goes to a list, what
// equals it to another, some more than k elements as a rule, and they are ranked by
// counting (hundreds of them, in rows of falling order, by k maxima).  Places decide
// between equal logits all the way.  Where more elements equal the k-th stripe's first
// than the list holds (rows of which all but a few logits are -inf, or of equal logits)
// the first of them are looked for from the start of the part.  Only a row made for it
// (more than a thousand larger elements in those stripes) overflows the list of the
// others: then the stripes are read k times.
//
// A row is split over a cluster of CTAs, which hand their parts to the first of them
// through its shared memory: no workspace, no second launch.  The CTAs stay for as
// many rows as fall to them; a warp of each copies the rows' next pieces into a ring
// meanwhile (40 KB, four CTAs on an SM), so that memory is read on while a row's last
// steps, which are rounds of latency, are taken.
//
// Rows of 151936 on 608 CTAs: 1088 of bf16 with k = 5 in 78 us (330 MB, 4.2 TB/s; 72
// with k = 0: two rows fall to most CTAs and one to some, which is 11 us of it), 190 of
// fp32 among 272 with k = 20 in 33 us (115 MB, 3.5 TB/s; 380 parts, of which two fall to
// some SMs and three to others), of which some 6 are the start and the selection.  With a
// launch's CTAs for each part instead, without the ring: 97 and 50.  With k = 20, 600 rows
// of bf16: 53 us, with 50 logits left by a filter 71, of equal logits 64, sorted 54 (with
// one list of 512 for all candidates 52, 69, 1490, 1455; 64 rows 19, 39, 35 and 29, and 19,
// 221, 221 and 203).
#include <algorithm>
#include <cstddef>

#include "barrier_wait.cuh"
#include "lsp_internal.h"
#include "q4.cuh"

namespace lsp {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;      // that add up; a warp more loads, and one joins a row's parts
constexpr int kMaxCluster = 8;
constexpr int kPerSm = 4;
constexpr int kPieceBytes = 64;                  // of a row, for a thread at a time
constexpr int kStages = 5, kStageBytes = kThreads * kPieceBytes;
constexpr int kStripes = kThreads;               // of a CTA's part: stripe i, of thread i, has its pieces i, i + kStripes, ...
// Candidates of a CTA: elements above the cut, of k pieces of 64 bytes (and the singles of as many threads) as a rule, and
// places of elements that equal it.
constexpr int kList = kLogprobsMaxK * 33, kTies = 256;
constexpr int kFew = 256;                        // of the list, that are ranked by counting
constexpr uint32_t kWhole = 0x80000000u;         // of a stripe: all of it is read again
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLeast = -150.0f;                // 2^t is 0 from here on
constexpr float kLowest = -3.402823466e38f;

// What a CTA has of a row, in the shared memory of its cluster's first.
struct Partial {
  float m, s, a;
  unsigned long long sorted[kLogprobsMaxK];      // its k largest elements: key and place, 0: none
};

struct Smem {
  alignas(128) uint8_t ring[kStages][kStageBytes];
  Partial part[2][kMaxCluster];                  // by turns
  unsigned long long list[kList + kTies];        // above the cut; equal to it
  unsigned long long sorted[kLogprobsMaxK];
  uint32_t stripe[kStripes];
  float red[kWarps];
  float2 red2[kWarps];
  unsigned long long best[kWarps];
  uint32_t least[kWarps];
  uint64_t full[kStages], empty[kStages];
  uint64_t parts[2], taken[2];                   // the cluster's parts of a row are there; the first has read them
  int count[2], stripes, abort;                  // of the lists
};
static_assert(kPerSm * (sizeof(Smem) + 128 + 1024) <= 228 * 1024, "CTAs of an SM");

__device__ __forceinline__ float ex2a(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Whole numbers of a type's width that order as its logits do (-0 as 0; NaN below all); 0 stands for no element.
template <typename T>
constexpr int kKeyBits = 8 * (int)sizeof(T);
template <typename T>
__device__ __forceinline__ uint32_t key_of(float x) {
  if (x != x) return 1u;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (u & 0x80000000u ? ~u : u | 0x80000000u) >> (32 - kKeyBits<T>);
}
template <typename T>
__device__ __forceinline__ float of_key(uint32_t k) {
  k <<= 32 - kKeyBits<T>;
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k & (sizeof(T) == 2 ? 0xFFFF0000u : 0xFFFFFFFFu));
}
// Key and place in one: the larger, and of equal ones the first, is the larger.
__device__ __forceinline__ unsigned long long entry(uint32_t key, uint32_t at) { return (unsigned long long)key << 32 | ~at; }

template <typename T>
struct Piece {
  static constexpr int kElems = kPieceBytes / (int)sizeof(T), kOf = 16 / (int)sizeof(T);
  uint4 v[4];
  __device__ __forceinline__ void unpack(int q, float* x) const {        // its q-th 16 bytes
    const uint32_t w[4] = {v[q].x, v[q].y, v[q].z, v[q].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      } else {
        x[i] = __uint_as_float(w[i]);
      }
    }
  }
  __device__ __forceinline__ float top() const { // the largest, NaN aside
    float t;
    if constexpr (sizeof(T) == 2) {
      __nv_bfloat162 m[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) m[q] = __hmax2(__hmax2(bits_bf2(v[q].x), bits_bf2(v[q].y)), __hmax2(bits_bf2(v[q].z), bits_bf2(v[q].w)));
      const __nv_bfloat162 a = __hmax2(__hmax2(m[0], m[1]), __hmax2(m[2], m[3]));
      t = fmaxf(__low2float(a), __high2float(a));
    } else {
      t = -INFINITY;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float x[4];
        unpack(q, x);
        t = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), t);
      }
    }
    return t;
  }
};

// A CTA's part of a row, in places: the row's elements before its first 16-byte
// boundary (place tid < head), the part's pieces from there on (places kStripes + i),
// and the elements behind the last piece (from place `tail_at` on).  Places rise with
// the index.
template <typename T>
struct Part {
  const T* z;
  int head, body, first, pieces, tail, tail_at;  // body: index of the row's first piece; first: of the part's, in pieces
  int tail_index;
  __device__ __forceinline__ uint4 quarter(int i, int q) const { return __ldcg(reinterpret_cast<const uint4*>(z + body) + 4 * (int64_t)(first + i) + q); }
  __device__ __forceinline__ int index(int i) const { return body + (first + i) * Piece<T>::kElems; }   // of a piece's first element
};

struct Scale {
  float c, inv;         // log2(e) / T, its reciprocal
  float large;          // logits up to here: t is finite, and what ref rounds off below 2^-4
};

// Of a thread's elements: the largest of those that have been m, and sums of 2^t and
// 2^t t with t = z c - ref, ref = m c rounded (what that rounds off is the same for all
// and is taken back at the end); of its stripe the largest logit, its piece's place,
// and the largest of the other pieces.
struct Stats {
  float m, ref;
  float least;          // logits below count nothing and are raised to here; NaN: t = (z - m) c, limited, one by one
  uint32_t low;         // the same as a pair of bf16, rounded down
  float2 s, a;          // of every other element, to be added
  float best, other;
  uint32_t place;
};

// The sums move to a higher m when an element, `top`, exceeds theirs by 2^8 (they are
// fp32: what is added meanwhile loses nothing).  They are relative to ref, or where least is NaN to m itself, and so
// afterwards; single: to m.
__device__ __forceinline__ void raise(Stats& st, float top, const Scale& k, bool single) {
  if (!((top - st.m) * k.c > 8.0f)) return;
  const bool was = st.least == st.least, fine = !single && fabsf(top) <= k.large;
  const float ref = top * k.c;
  float t = was && fine ? st.ref - ref : (st.m - top) * k.c;
  if (was && !fine) t -= fmaf(st.m, k.c, -st.ref);
  if (!was && fine) t += fmaf(top, k.c, -ref);
  t = max_nan(t, kLeast);
  const float r = ex2a(t);
  st.a = make_float2(r * (st.a.x + st.s.x * t), r * (st.a.y + st.s.y * t));
  st.s = make_float2(r * st.s.x, r * st.s.y);
  st.m = top;
  st.ref = ref;
  // (200 / c below m, which is 10^6 / c at most: many of its last places)
  st.least = fine ? top - 200.0f * k.inv : __uint_as_float(0x7FC00000u);
  const __nv_bfloat16 low = __float2bfloat16_rd(st.least);
  st.low = bf2_bits(__halves2bfloat162(low, low));
}
__device__ __forceinline__ void add_limited(Stats& st, float x, const Scale& k) {
  const float t = max_nan((x - st.m) * k.c, kLeast), e = ex2a(t);
  st.s.x += e;
  st.a.x = fmaf(e, t, st.a.x);
}

// A piece at `place`.  As long as m stays within +-large, every t is finite, and e t = 0
// where e = 0: what is far below (-inf, a banned token) is raised to where e is 0 already.
template <typename T>
__device__ __forceinline__ void add_piece(Stats& st, Piece<T>& v, uint32_t place, const Scale& k) {
  const float top = v.top();
  st.other = fmaxf(st.other, fminf(top, st.best));
  if (top > st.best) st.best = top, st.place = place;
  raise(st, top, k, false);
  if (st.least != st.least) {                    // nothing but -inf so far, or logits too large
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float x[Piece<T>::kOf];
      v.unpack(q, x);
#pragma unroll
      for (int i = 0; i < Piece<T>::kOf; ++i) add_limited(st, x[i], k);
    }
    return;
  }
  const float2 c = make_float2(k.c, k.c), ref = make_float2(-st.ref, -st.ref);
  const __nv_bfloat162 low2 = bits_bf2(st.low);
  float2 s[2] = {st.s, {0.f, 0.f}}, a[2] = {st.a, {0.f, 0.f}};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float x[Piece<T>::kOf];
    if constexpr (sizeof(T) == 2) {
      v.v[q] = make_uint4(bf2_bits(__hmax2_nan(bits_bf2(v.v[q].x), low2)), bf2_bits(__hmax2_nan(bits_bf2(v.v[q].y), low2)),
                          bf2_bits(__hmax2_nan(bits_bf2(v.v[q].z), low2)), bf2_bits(__hmax2_nan(bits_bf2(v.v[q].w), low2)));
      v.unpack(q, x);
    } else {
      v.unpack(q, x);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = max_nan(x[i], st.least);
    }
#pragma unroll
    for (int i = 0; i < Piece<T>::kOf; i += 2) {
      const float2 t = fma2(make_float2(x[i], x[i + 1]), c, ref), e = make_float2(ex2a(t.x), ex2a(t.y));
      s[(i >> 1) & 1] = add2(s[(i >> 1) & 1], e);
      a[(i >> 1) & 1] = fma2(e, t, a[(i >> 1) & 1]);
    }
  }
  st.s = add2(s[0], s[1]);
  st.a = add2(a[0], a[1]);
}
// The pieces are over: sums relative to m.
__device__ __forceinline__ void settle(Stats& st, const Scale& k) {
  if (st.least != st.least) return;
  const float off = fmaf(st.m, k.c, -st.ref), f = ex2a(-off);
  st.a = make_float2(f * (st.a.x - off * st.s.x), f * (st.a.y - off * st.s.y));
  st.s = make_float2(f * st.s.x, f * st.s.y);
  st.least = __uint_as_float(0x7FC00000u);
}
// A single element, behind that.
__device__ __forceinline__ void add_one(Stats& st, float x, const Scale& k) {
  raise(st, x, k, true);
  add_limited(st, x, k);
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Among the threads that add up.
__device__ __forceinline__ void meet() { named_bar(1, kThreads); }
__device__ __forceinline__ int count_all(bool x) {
  int n;
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.popc.aligned.u32 %0, 1, %2, p;\n}"
      : "=r"(n)
      : "r"((uint32_t)x), "n"(kThreads)
      : "memory");
  return n;
}

__device__ __forceinline__ unsigned long long block_max(unsigned long long v, Smem& sm) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  meet();
  if (lane == 0) sm.best[warp] = v;
  meet();
  v = sm.best[lane & (kWarps - 1)];
#pragma unroll
  for (int o = kWarps / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// sm.sorted = the k largest elements of the part (0 where it has fewer); head, tail: this thread's single elements.
template <typename T>
__device__ __forceinline__ void part_top(const Part<T>& part, const Stats& st, float head, float tail, int k, Smem& sm) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool some = tid < part.head || tid < part.pieces || tid < part.tail;
  const uint32_t key = some ? key_of<T>(st.best) : 0u;
  if (tid == 0) sm.count[0] = sm.count[1] = sm.stripes = 0;
  if (tid < k) sm.sorted[tid] = 0;
  // the largest `cut` that k stripes reach, bit by bit; among equal ones, the place that makes them k
  uint32_t cut = 0, last = 0xFFFFFFFFu;
  int reach = kStripes;
  for (uint32_t bit = 1u << (kKeyBits<T> - 1); bit; bit >>= 1) {
    const int n = count_all(key >= (cut | bit));
    if (n >= k) {
      cut |= bit;
      reach = n;
      if (n == k) break;
    }
  }
  if (reach == k) {                              // the least of theirs
    const uint32_t least = __reduce_min_sync(0xffffffffu, key >= cut ? key : 0xFFFFFFFFu);
    if (lane == 0) sm.least[warp] = least;
    meet();
    cut = __reduce_min_sync(0xffffffffu, sm.least[lane & (kWarps - 1)]);
  } else if (cut > 0) {
    last = 0;                                    // places below it leave less than k stripes
    for (uint32_t bit = 1u << (31 - __clz(part.tail_at + kStripes)); bit; bit >>= 1)
      if (count_all(key > cut || (key == cut && st.place < (last | bit))) < k) last |= bit;
  }
  auto in = [&](uint32_t e_key, uint32_t place) { return e_key > cut || (e_key == cut && place <= last); };
  const float least = of_key<T>(cut);            // (most elements are below it, and go no further)
  auto put = [&](float x, uint32_t place, int index) {
    if (cut > 0 && !(x >= least)) return;
    const uint32_t e = key_of<T>(x);
    if (!in(e, place)) return;
    const int tie = e == cut, at = atomicAdd(&sm.count[tie], 1);
    if (at < (tie ? kTies : kList)) sm.list[at + (tie ? kList : 0)] = entry(e, (uint32_t)index);
  };
  auto load_piece = [&](int i) {
    Piece<T> v;
#pragma unroll
    for (int q = 0; q < 4; ++q) v.v[q] = part.quarter(i, q);
    return v;
  };
  auto each = [&](const Piece<T>& v, int i, auto f) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float x[Piece<T>::kOf];
      v.unpack(q, x);
#pragma unroll
      for (int e = 0; e < Piece<T>::kOf; ++e) f(x[e], part.index(i) + q * Piece<T>::kOf + e);
    }
  };
  auto put_piece = [&](const Piece<T>& v, int i) {
    each(v, i, [&](float x, int index) { put(x, kStripes + i, index); });
  };
  const bool mine = some && in(key, st.place);
  if (mine) {
    if (tid < part.head) put(head, tid, tid);
    if (tid < part.tail) put(tail, part.tail_at + tid, part.tail_index + tid);
    // (another piece with the largest logit lies behind, and has the place to decide; a single element counts as a piece)
    const uint32_t other = key_of<T>(st.other);
    if (other >= cut) sm.stripe[atomicAdd(&sm.stripes, 1)] = tid | (other > cut ? kWhole : 0u);
    if ((other < cut || (other == cut && st.place > last)) && st.place >= kStripes && st.place < (uint32_t)part.tail_at)
      put_piece(load_piece((int)st.place - kStripes), (int)st.place - kStripes);
  }
  meet();
  // a warp takes stripes in turn, a lane every 32nd piece; where the others equal the cut, up to the last place that counts
  const int stripes = sm.stripes, tied = last < kStripes ? 0 : (int)min((uint32_t)part.pieces, last - kStripes + 1);
  for (int x = warp; x < stripes; x += kWarps) {
    const uint32_t stripe = sm.stripe[x];
    const int upto = stripe & kWhole ? part.pieces : tied;
    for (int i = lane * kStripes + (int)(stripe & ~kWhole); i < upto; i += 32 * kStripes) put_piece(load_piece(i), i);
  }
  meet();
  const int n = sm.count[0], ties = sm.count[1];
  if (n <= kFew) {
    // those that equal the cut behind the others
    const int all = ties <= kTies ? n + ties : n;
    for (int i = tid; i < all; i += kThreads) {
      const bool tie = i >= n;
      const unsigned long long* list = sm.list + (tie ? kList : 0);
      const int len = tie ? ties : n;
      const unsigned long long x = list[tie ? i - n : i];
      int rank = tie ? n : 0;
      for (int j = 0; j < len; ++j) rank += list[j] > x;
      if (rank < k) sm.sorted[rank] = x;
    }
    if (n < k && ties > kTies) {
      // more of them than the list holds (most of a filtered row, or one of equal logits): in the order of their index, as
      // far as it takes
      int found = n;
      auto take = [&](uint32_t which, int index) {         // which: of this thread's next elements, from `index` on
        const int count = __popc(which);
        int before = count;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int x = __shfl_up_sync(0xffffffffu, before, o);
          if (lane >= o) before += x;
        }
        meet();
        if (lane == 31) sm.least[warp] = before;
        meet();
        int rank = found + before - count;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const int x = (int)sm.least[w];
          if (w < warp) rank += x;
          found += x;
        }
        for (; which && rank < k; which &= which - 1) sm.sorted[rank++] = entry(cut, (uint32_t)(index + __ffs(which) - 1));
      };
      take(tid < part.head && key_of<T>(head) == cut, tid);
      for (int i0 = 0; i0 < part.pieces && found < k; i0 += kThreads) {
        const int i = i0 + tid;
        uint32_t which = 0;
        if (i < part.pieces) each(load_piece(i), i, [&](float x, int index) { which |= (uint32_t)(x == least) << (index - part.index(i)); });
        take(which, part.index(i));
      }
      if (found < k) take(tid < part.tail && key_of<T>(tail) == cut, part.tail_index + tid);
    }
    meet();
    return;
  }
  // one alternative at a time, of the list, or of the stripes' elements where it overflows
  if (tid == 0) sm.stripes = 0;
  meet();
  if (mine) sm.stripe[atomicAdd(&sm.stripes, 1)] = tid;
  meet();
  unsigned long long before = ~0ull;
  for (int r = 0; r < k; ++r) {
    unsigned long long best = 0;
    auto see = [&](float x, int index) {
      const unsigned long long e = entry(key_of<T>(x), (uint32_t)index);
      if (e < before && e > best) best = e;
    };
    if (n <= kList) {
      for (int i = tid; i < n; i += kThreads) {
        const unsigned long long e = sm.list[i];
        if (e < before && e > best) best = e;
      }
    } else {
      if (mine && tid < part.head) see(head, tid);
      for (int x = warp; x < sm.stripes; x += kWarps)
        for (int i = lane * kStripes + (int)sm.stripe[x]; i < part.pieces; i += 32 * kStripes) each(load_piece(i), i, see);
      if (mine && tid < part.tail) see(tail, part.tail_index + tid);
    }
    best = block_max(best, sm);
    if (tid == 0) sm.sorted[r] = best;
    before = best;
    if (best == 0) break;
  }
  meet();
}

// The rows with a token that fall to cluster `mine` of `clusters`, in order; for whole warps.
struct Rows {
  const int32_t* tokens;
  int rows, V, clusters;
  int skip;                                      // rows with a token until the next of this cluster's
  int at = 0, token = -1;                        // the next 32 rows; token: of the lane's row
  unsigned left = 0;
  __device__ __forceinline__ bool valid(int t) const { return t >= 0 && t < V; }
  __device__ __forceinline__ int next(int* of) { // -1: no more
    for (;;) {
      const int n = __popc(left);
      if (n > skip) {
        for (; skip > 0; --skip) left &= left - 1;
        const int lane = __ffs(left) - 1;
        left &= left - 1;
        skip = clusters - 1;
        *of = __shfl_sync(0xffffffffu, token, lane);
        return at - 32 + lane;
      }
      skip -= n;
      if (at >= rows) return -1;
      const int r = at + (threadIdx.x & 31);
      token = r < rows ? tokens[r] : -1;
      left = __ballot_sync(0xffffffffu, valid(token));
      at += 32;
    }
  }
};

template <typename T>
__device__ __forceinline__ Part<T> part_of(const LogprobsParams& p, int row, int rank, int cluster) {
  constexpr int VE = Piece<T>::kElems;
  Part<T> part;
  part.z = static_cast<const T*>(p.z) + (int64_t)row * p.ld;
  const int off = (int)((16 - (reinterpret_cast<uintptr_t>(part.z) & 15)) & 15) / (int)sizeof(T);
  part.body = min(off, p.V);
  const int pieces = (p.V - part.body) / VE, per = (pieces + cluster - 1) / cluster;
  part.first = min(rank * per, pieces);
  part.pieces = min(per, pieces - part.first);
  part.head = rank == 0 ? part.body : 0;
  part.tail_index = part.body + pieces * VE;
  part.tail = rank == cluster - 1 ? p.V - part.tail_index : 0;
  part.tail_at = ((part.pieces + kStripes - 1) / kStripes + 1) * kStripes;
  return part;
}

template <typename T>
__device__ __forceinline__ void load_role(const LogprobsParams& p, Smem& sm, Rows rows, int rank, int cluster) {
  Place ring = {0, 1};                           // (the first uses wait for nobody)
  int token;
  for (int row = rows.next(&token); row >= 0; row = rows.next(&token)) {
    const Part<T> part = part_of<T>(p, row, rank, cluster);
    const char* from = reinterpret_cast<const char*>(part.z + part.body) + (int64_t)part.first * kPieceBytes;
    for (int i = 0; i < part.pieces; i += kThreads, ring.next(kStages)) {
      const uint32_t bar = smem_u32(&sm.full[ring.stage]), bytes = min(part.pieces - i, kThreads) * kPieceBytes;
      if (!tc_wait(smem_u32(&sm.empty[ring.stage]), ring.phase, &sm.abort, p.err)) return;
      if ((threadIdx.x & 31) == 0) {
        mbar_expect_tx(bar, bytes);
        bulk_load(smem_u32(sm.ring[ring.stage]), from + (int64_t)i * kPieceBytes, bytes, bar);
      }
      __syncwarp();
    }
  }
}

// Shared memory of the cluster's CTA `rank`, and its barriers.
__device__ __forceinline__ uint32_t in_cta(uint32_t at, int rank) {
  uint32_t x;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(x) : "r"(at), "r"(rank));
  return x;
}
__device__ __forceinline__ void store_far(uint32_t at, unsigned long long x) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(x) : "memory");
}
__device__ __forceinline__ void arrive_far(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
struct ClusterWait : BarrierWait {
  __device__ __forceinline__ bool ready() const {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
  }
};

template <typename T>
__device__ __forceinline__ void add_role(const LogprobsParams& p, Smem& sm, Rows rows, int rank, int cluster) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float c = kLog2e / p.temperature;
  const Scale scale = {c, p.temperature * 0.69314718055994531f, fminf(1e38f, 1e6f / c)};
  // A wait that gives up leaves the row wrong, but its steps are taken all the same: the barriers of the CTA have no
  // limit, so its threads leave together, behind a row.
  bool failed = false;
  auto wait = [&](uint64_t* bar, uint32_t parity) { failed |= !tc_wait(smem_u32(bar), parity, &sm.abort, p.err); };
  Place ring = {0, 0};
  const uint32_t ring_at = smem_u32(sm.ring) + tid * kPieceBytes, zero = (uint32_t)p.V >> 31;
  int token;
  uint32_t turn = 0;
  for (int row = rows.next(&token); row >= 0; row = rows.next(&token), ++turn) {
    const Part<T> part = part_of<T>(p, row, rank, cluster);
    float head = 0.f, tail = 0.f;
    if (tid < part.head) head = to_f(part.z[tid]);
    if (tid < part.tail) tail = to_f(part.z[part.tail_index + tid]);
    Stats st = {kLowest, kLowest, __uint_as_float(0x7FC00000u), 0u, {0.f, 0.f}, {0.f, 0.f}, -INFINITY, -INFINITY, 0u};
    // (a thread's first place, for stripes of -inf alone)
    st.place = tid < part.head ? tid : tid < part.pieces ? kStripes + tid : part.tail_at + tid;
    for (int i0 = 0; i0 < part.pieces; i0 += kThreads, ring.next(kStages)) {
      wait(&sm.full[ring.stage], ring.phase);
      Piece<T> v;
      // (eight lanes, 64 bytes apart, read eight different 16 bytes of 128; the order within a piece does not matter)
#pragma unroll
      for (int q = 0; q < 4; ++q) v.v[q] = ld_shared4(ring_at + ring.stage * kStageBytes + ((q + (lane >> 1)) & 3) * 16);
      if (i0 + tid < part.pieces) add_piece(st, v, kStripes + i0 + tid, scale);
      // (the sum needs all of the piece; as soon as the loads are there, in front of the piece, is 1 % slower)
      arrive_after_reads(smem_u32(&sm.empty[ring.stage]), __float_as_uint(st.s.x), zero);
    }
    settle(st, scale);
    if (tid < part.head) {                       // (the first of its stripe: it goes before an equal one)
      st.other = fmaxf(st.other, fminf(head, st.best));
      if (head >= st.best) st.best = head, st.place = tid;
      add_one(st, head, scale);
    }
    if (tid < part.tail) {
      st.other = fmaxf(st.other, fminf(tail, st.best));
      if (tail > st.best) st.best = tail, st.place = part.tail_at + tid;
      add_one(st, tail, scale);
    }
    // the CTA's sums
    const float wm = warp_max(st.m);
    if (lane == 0) sm.red[warp] = wm;
    meet();
    float m = sm.red[lane & (kWarps - 1)];
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    {
      const float t = max_nan((st.m - m) * c, kLeast), r = ex2a(t), s = st.s.x + st.s.y;
      const float ws = warp_sum(r * s), wa = warp_sum(r * (st.a.x + st.a.y + s * t));
      if (lane == 0) sm.red2[warp] = make_float2(ws, wa);
    }
    if (p.k > 0) part_top<T>(part, st, head, tail, p.k, sm); else meet();
    // ... to the first CTA (its place is free once the row before the last is joined)
    if (warp == 0) {
      const uint32_t mine = smem_u32(&sm.part[turn & 1][rank]), far = in_cta(mine, 0);
      failed |= !warp_wait(ClusterWait{{smem_u32(&sm.taken[turn & 1]), ((turn >> 1) & 1) ^ 1, &sm.abort, p.err}}, kWaitLimitNs);
      if (lane == 0) {
        float s = 0.f, a = 0.f;
        for (int w = 0; w < kWarps; ++w) s += sm.red2[w].x, a += sm.red2[w].y;
        store_far(far, (unsigned long long)__float_as_uint(s) << 32 | __float_as_uint(m));
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(far + 8), "f"(a) : "memory");
      }
      if (lane < p.k) store_far(far + (uint32_t)offsetof(Partial, sorted) + 8 * lane, sm.sorted[lane]);
      arrive_far(in_cta(smem_u32(&sm.parts[turn & 1]), 0));      // (every lane, for what it has stored)
    }
    if (count_all(failed) > 0) break;            // (and the row's lists are read)
  }
}

// The warp of a cluster's first CTA that joins the parts of a row.
template <typename T>
__device__ __forceinline__ void join_role(const LogprobsParams& p, Smem& sm, Rows rows, int cluster) {
  const int lane = threadIdx.x & 31;
  const float c = kLog2e / p.temperature;
  const float nan = __uint_as_float(0x7FC00000u);
  int token;
  uint32_t turn = 0;
  for (int row = rows.next(&token); row >= 0; row = rows.next(&token), ++turn) {
    const float z = to_f(static_cast<const T*>(p.z)[(int64_t)row * p.ld + token]);
    if (!warp_wait(ClusterWait{{smem_u32(&sm.parts[turn & 1]), (turn >> 1) & 1, &sm.abort, p.err}}, kWaitLimitNs)) return;
    const Partial* all = sm.part[turn & 1];
    float top = kLowest;
    for (int r = 0; r < cluster; ++r) top = fmaxf(top, all[r].m);
    float s = 0.f, a = 0.f;
    for (int r = 0; r < cluster; ++r) {
      const float t = max_nan((all[r].m - top) * c, kLeast), x = ex2a(t);
      s += x * all[r].s;
      a += x * (all[r].a + all[r].s * t);
    }
    const bool none = !(s > 0.f) || !isfinite(top);              // no distribution
    const float ln_s = logf(s);
    if (lane == 0) {
      // (S may come out below 1 by what its terms are rounded)
      p.logprob[row] = none ? nan : fminf((z - top) / p.temperature - ln_s, 0.f);
      if (p.entropy) p.entropy[row] = none ? nan : fmaxf(ln_s - a / s * 0.69314718055994531f, 0.f);
    }
    // lane r has the first that is left of part r's list; the largest of those goes to lane i in round i
    uint32_t key = 0, at = 0, won_key = 0, won_at = 0;
    int next = 0;
    auto pull = [&]() {
      const unsigned long long x = lane < cluster && next < p.k ? all[lane].sorted[next] : 0;
      key = (uint32_t)(x >> 32);
      at = (uint32_t)x;
      ++next;
    };
    pull();
    for (int i = 0; i < p.k; ++i) {
      const uint32_t k = __reduce_max_sync(0xffffffffu, key), w = __reduce_max_sync(0xffffffffu, key == k ? at : 0u);
      if (lane == i) won_key = k, won_at = w;
      if (key == k && at == w) pull();
    }
    if (lane < p.k) {                            // (k <= V: there are k elements)
      const int64_t to = (int64_t)row * p.k + lane;
      if (p.top) p.top[to] = none ? -1 : (int)~won_at;
      if (p.top_logprob) p.top_logprob[to] = none ? nan : fminf((of_key<T>(won_key) - top) / p.temperature - ln_s, 0.f);
    }
    __syncwarp();
    if (lane < cluster) arrive_far(in_cta(smem_u32(&sm.taken[turn & 1]), lane));
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads + 64, kPerSm) logprobs_kernel(const LogprobsParams p, int cluster) {
  extern __shared__ uint8_t raw[];
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(raw) + 127) & ~static_cast<uintptr_t>(127));
  const int tid = threadIdx.x, rank = blockIdx.x % cluster;
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem_u32(&sm.full[i]), 1);
      mbar_init(smem_u32(&sm.empty[i]), kWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sm.parts[i]), 32 * cluster);
      mbar_init(smem_u32(&sm.taken[i]), 1);
    }
    sm.abort = 0;
    fence_barrier_init();
  }
  cluster_sync();                                // (barriers are there before another CTA arrives at them)
  griddep_wait();
  griddep_launch();
  const Rows rows{p.tokens, p.rows, p.V, (int)gridDim.x / cluster, (int)blockIdx.x / cluster};
  if (tid >= kThreads + 32) {
    if (rank == 0) join_role<T>(p, sm, rows, cluster);
  } else if (tid >= kThreads) {
    load_role<T>(p, sm, rows, rank, cluster);
  } else {
    // rows without a token
    for (int r = blockIdx.x * kThreads + tid; r < p.rows; r += gridDim.x * kThreads) {
      const int token = p.tokens[r];
      if (rows.valid(token)) continue;
      for (int i = 0; i < p.k; ++i) {
        if (p.top) p.top[(int64_t)r * p.k + i] = -1;
        if (p.top_logprob) p.top_logprob[(int64_t)r * p.k + i] = -INFINITY;
      }
      p.logprob[r] = -INFINITY;
      if (p.entropy) p.entropy[r] = 0.f;
      if (token != -1) set_err(p.err, LSP_DEV_BAD_TOKEN);
    }
    add_role<T>(p, sm, rows, rank, cluster);
  }
  __syncthreads();
  // Every load has been waited for, unless a wait gave up: then loads may still be landing, and the CTA stays for
  // them (bounded).
  if (*reinterpret_cast<volatile int*>(&sm.abort) && tid == 0) {
    const uint64_t t0 = global_ns();
    while (global_ns() - t0 < 1000000ull) {}
  }
  cluster_sync();                                // (nobody stores into a CTA that is gone)
}

// CTAs of a row: a part costs some 5 us besides reading it, so no more than fill the GPU's SMs more than twice over
// (rows of 151936, k = 20: 190 of fp32 43, 38, 43 and 44 us with 1, 2, 4 and 8; 500 76, 77, 81, 89; 64 31, 23, 20, 20),
// while each has a round of loads.
int choose_cluster(int rows, int V, int es, int num_sms) {
  const int64_t pieces = (int64_t)V * es / kPieceBytes;
  int n = 1;
  while (n < kMaxCluster && (int64_t)rows * n * 5 < 12 * num_sms && pieces > (int64_t)kThreads * n) n *= 2;
  return n;
}

template <typename T>
int launch(const LogprobsParams& p, int num_sms, cudaStream_t s) {
  static bool set[8] = {};
  const int smem = (int)sizeof(Smem) + 128;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return LSP_ERR_CUDA;
  if (dev >= 8 || !set[dev]) {
    if (cudaFuncSetAttribute(logprobs_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return LSP_ERR_CUDA;
    if (dev < 8) set[dev] = true;
  }
  const int cluster = choose_cluster(p.rows, p.V, (int)sizeof(T), num_sms);
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads + 64);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  // as many clusters as run at once: what is left over would come behind all the others' rows
  static int most[8][4] = {};
  const int log = 31 - __builtin_clz(cluster);
  int at_once = dev < 8 ? most[dev][log] : 0;
  if (at_once == 0) {
    cfg.gridDim = dim3((unsigned)(kPerSm * num_sms / cluster * cluster));
    if (cudaOccupancyMaxActiveClusters(&at_once, logprobs_kernel<T>, &cfg) != cudaSuccess || at_once < 1) return LSP_ERR_CUDA;
    if (dev < 8) most[dev][log] = at_once;
  }
  cfg.numAttrs = 2;
  cfg.gridDim = dim3((unsigned)(std::min(p.rows, at_once) * cluster));
  return cudaLaunchKernelEx(&cfg, logprobs_kernel<T>, p, cluster) == cudaSuccess ? LSP_OK : LSP_ERR_CUDA;
}

}  // namespace

int launch_logprobs(const LogprobsParams& p, int dtype, int num_sms, cudaStream_t s) {
  return dtype == LSP_DTYPE_BF16 ? launch<bf16>(p, num_sms, s) : launch<float>(p, num_sms, s);
}

}  // namespace lsp
