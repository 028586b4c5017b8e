// Work distribution of the shared-prefix attention.
//
// Query rows.  The rep = nq/nkv query heads of a KV head score the same keys,
// so a row of a tile is (token, head of the group): a tile holds tok_tile =
// tile rows / rep tokens, a unit kUnit tiles that share the keys they load.
//
// Shared part: the whole pages before every row's position that all sequences
// hold, `base` tokens.  All `total` tokens of the batch are stacked into units
// against them, without regard to whose they are (nothing is masked), and the
// keys are cut into `splits` ranges: items (head, range, unit), the unit fastest.
//
// Own part: tokens [base, len) of each sequence, its own rows only, causal: items
// (sequence, unit, head).
//
// As many shared items as go round evenly are dealt to the CTAs whole, in turn,
// so that units of the same keys run at the same time and find each other's
// loads in L2.  The rest of them and the own items form one line, each as long
// as it costs, that is cut into a piece of the same length for every CTA.  A
// piece may start and end inside an item.  A CTA goes through the shared segments
// of its piece from the last to the first: with pieces somewhat shorter than
// items, it then comes to the first keys of one item and the last of the item
// before when the others do (forwards, nearly every unit read the keys from
// memory: 4.7 GB instead of 1.1 at 32 requests over 128K, 0.92 ms instead of 0.80).
//
// Every segment (the part of an item that one CTA has) leaves unnormalised sums
// and the running maximum and sum of its rows in rows of the workspace; a second
// kernel joins a row's segments, which it finds by the same arithmetic.  A
// segment of the line lies at (rows of the items before it) + CTA * (rows of a
// unit), which no two share: along the line the item or the CTA rises from
// segment to segment, each by at least the room of one.
#pragma once

#include <climits>

#include "common.cuh"
#include "lsp_internal.h"

namespace lsp {

struct PrefixSched {
  int base;             // tokens of the shared part
  int blocks;           // its key blocks,
  int range, longer;    // of a key range; the first `longer` ranges have one more
  int items, whole;     // shared items; those dealt whole, the first ones
  int len_two, len_last;    // lengths of the shared items of a range's units: all but the last, the last
  int64_t len_range;    // of a range's items together
  int64_t whole_line;   // of the items dealt whole
  int64_t shared_line;  // of the other shared items: where own items begin on the line
  int64_t line;         // length of the line
  int ctas;             // pieces it is cut into: CTAs [0, ctas) have one
  int together;         // key blocks that a cut keeps together in a short item
};

// A kernel's tiles of a unit and keys of a block, and what work costs a CTA of it, for
// dealing it out, in units of 0.37 us: a key block against few and against many rows (more
// than kFewRows; 0: than a tile's), and what a segment takes besides.  (Constants: as
// parameters, with the join's divisions by them, attention of 16 requests of one row over
// 32K took 49.3 us instead of 47.8.)
//
// A segment of the tensor cores costs as much as two blocks, so a cut leaves four
// together in a short item (of up to kShort), unless there is less work than CTAs;
// a block of the other kernels takes longer than what comes with it.
template <int kUnitTiles_, int kBlock_, int kFewRows_, int kFew_, int kMany_, int kSegment_>
struct PrefixWork {
  static constexpr int kUnitTiles = kUnitTiles_, kBlock = kBlock_, kFewRows = kFewRows_, kFew = kFew_, kMany = kMany_, kSegment = kSegment_;
};
// one row tile 1.1 us a block, two 1.46, a segment 1.9 (16 requests over 32K)
using TcWork = PrefixWork<kPrefixTcTiles, kPrefixTcKeys, 0, 3, 4, 5>;
// over a cache in 4 bits both are as long as it takes to unpack a block (16 requests of 17 rows over 32K 172 us, with the
// costs of bf16 198, when they were chosen)
using TcQ4Work = PrefixWork<kPrefixTcTiles, kPrefixTcKeys, 0, 5, 5, 8>;
// unpacked again for every 8 rows (32 of one row over 8K and up to 4K of their own 52 us, with the costs below 76)
using Q4Work = PrefixWork<1, kPrefixQ4Keys, 8, 4, 10, 8>;
// (the fp32 kernel's warps have eight rows each, and those without rows leave the block to the others)
using FmaWork = PrefixWork<1, kPrefixFmaKeys, 32, 3, 4, 5>;

constexpr int kTogether = 4, kShort = 8;
template <class W>
__device__ __forceinline__ int block_cost(const PrefixAttnParams& p, int tokens) {
  return (W::kFewRows ? tokens * p.rep > W::kFewRows : tokens > p.tok_tile) ? W::kMany : W::kFew;
}
struct __align__(16) PrefixSeq {
  int seq, first, rows, len;    // row of the table (-1: none), first row of q, rows, tokens
};

// Division of what outgrows 32 bits only in the longest batches, kept out of line:
// the schedule runs once, and costs what its code takes to be fetched.
static __device__ __noinline__ int64_t long_div(int64_t a, int64_t b) { return a / b; }
__device__ __forceinline__ int cdiv(int a, int b) { return (a + b - 1) / b; }

// Sequence i of the batch; rows = 0 for one the call cannot use.  kFresh: read from
// memory whatever this grid has read there before.
template <bool kFresh>
__device__ __forceinline__ int seq_word(const int32_t* p) {
  return kFresh ? *reinterpret_cast<const volatile int32_t*>(p) : *p;
}
template <bool kFresh = false>
__device__ __forceinline__ PrefixSeq prefix_seq(const PrefixAttnParams& p, int i, bool report) {
  PrefixSeq r;
  r.seq = seq_word<kFresh>(p.seqs + i);
  r.first = seq_word<kFresh>(p.start + i);
  r.rows = seq_word<kFresh>(p.start + i + 1) - r.first;
  r.len = 0;
  const int most = p.max_pages * p.page;
  bool bad = r.first < 0 || r.rows < 0 || r.first > p.total - r.rows || r.seq < 0 || r.seq >= p.n_seqs;
  if (!bad) {
    r.len = seq_word<kFresh>(p.len + r.seq);
    bad = r.len < 0 || r.len > most;
  }
  if (bad) {
    if (report) set_err(p.err, LSP_DEV_BAD_SEQ);
    r.seq = -1;
    r.rows = r.len = 0;
  }
  return r;
}

// Whether memory still says what r was made of (one round of loads where the call can use the sequence).
__device__ __forceinline__ bool same_seq(const PrefixAttnParams& p, int i, const PrefixSeq& r) {
  if (r.seq >= 0) {
    const int seq = seq_word<true>(p.seqs + i), first = seq_word<true>(p.start + i), next = seq_word<true>(p.start + i + 1);
    return (seq == r.seq) & (first == r.first) & (next - first == r.rows) & (seq_word<true>(p.len + r.seq) == r.len);
  }
  const PrefixSeq x = prefix_seq<true>(p, i, false);
  return x.seq < 0 && x.first == r.first;
}

// Own key blocks that unit u of a sequence has to see.
template <class W>
__device__ __forceinline__ int own_blocks(const PrefixAttnParams& p, const PrefixSeq& r, int base, int u) {
  const int upto = min(r.rows, (u + 1) * W::kUnitTiles * p.tok_tile);
  return max(0, cdiv(r.len - r.rows + upto - base, W::kBlock));
}

__device__ __forceinline__ int own_units(const PrefixAttnParams& p, const PrefixSeq& r, int unit_tiles) {
  return cdiv(r.rows, unit_tiles * p.tok_tile);
}

// Length on the line of an own item of a unit with `blocks` key blocks:
template <class W>
__device__ __forceinline__ int item_length(const PrefixAttnParams& p, const PrefixSeq& r, int u, int blocks) {
  return blocks > 0 ? W::kSegment + blocks * block_cost<W>(p, r.rows - u * W::kUnitTiles * p.tok_tile) : 0;
}

// Built by one warp of every CTA; line_base [n + 1], info [n] in shared memory.
template <class W>
__device__ __forceinline__ PrefixSched build_sched(const PrefixAttnParams& p, int64_t* line_base, PrefixSeq* info, bool report) {
  const int lane = threadIdx.x & 31;
  PrefixSched s;
  int base = p.shared_len;
  bool any = false;
  for (int i = lane; i < p.n; i += 32) {
    const PrefixSeq r = prefix_seq(p, i, report);
    info[i] = r;
    if (r.rows > 0) base = min(base, r.len - r.rows);
    any |= r.rows > 0;
  }
  if (!__any_sync(0xffffffffu, any)) base = 0;   // rows of no sequence have nothing to see
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) base = min(base, __shfl_xor_sync(0xffffffffu, base, o));
  s.base = max(base, 0) / p.page * p.page;
  s.blocks = cdiv(s.base, W::kBlock);
  s.range = s.blocks / p.splits;
  s.longer = s.blocks - s.range * p.splits;
  s.items = s.blocks > 0 ? p.nkv * p.splits * p.units : 0;
  s.whole = s.items / p.grid * p.grid;
  const int most = s.range + (s.longer > 0);
  s.len_two = W::kSegment + most * W::kMany;
  s.len_last = W::kSegment + most * block_cost<W>(p, p.total - (p.units - 1) * W::kUnitTiles * p.tok_tile);
  s.len_range = (int64_t)(p.units - 1) * s.len_two + s.len_last;
  s.whole_line = (int64_t)(s.whole / p.units) * s.len_range + (int64_t)(s.whole % p.units) * s.len_two;
  s.shared_line = (int64_t)(s.items / p.units) * s.len_range - s.whole_line;
  int64_t line = 0;
  for (int i0 = 0; i0 < p.n; i0 += 32) {
    const int i = i0 + lane;
    int64_t mine = 0;
    if (i < p.n) {
      const PrefixSeq r = info[i];               // this lane's own store
      for (int u = 0, units = own_units(p, r, W::kUnitTiles); u < units; ++u)
        mine += item_length<W>(p, r, u, own_blocks<W>(p, r, s.base, u));
      mine *= p.nkv;
    }
    int64_t x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t a = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += a;
    }
    if (i < p.n) line_base[i] = line + x - mine;
    line += __shfl_sync(0xffffffffu, x, 31);
  }
  if (lane == 0) line_base[p.n] = line;
  s.line = s.shared_line + line;
  const int least = W::kFew;
  const bool small = s.line < (int64_t)p.grid * (W::kSegment + kTogether * least);
  s.together = W::kUnitTiles == 1 || small ? 1 : kTogether;
  s.ctas = small ? max(min((int)s.line / least, p.grid), 1) : p.grid;
  return s;
}

// Where CTA c's piece of the line begins (from c == ctas on: the line's end).
__device__ __forceinline__ int64_t piece_begin(const PrefixSched& s, int c) {
  if (c >= s.ctas) return s.line;
  return s.line < (1 << 21) ? (int64_t)((uint32_t)s.line * (uint32_t)c / (uint32_t)s.ctas) : long_div(s.line * c, s.ctas);   // c < 2^11
}
__device__ __forceinline__ int64_t div_floor(int64_t a, int64_t b) {           // a >= 0, b > 0
  return a <= INT_MAX && b <= INT_MAX ? (int64_t)((int)a / (int)b) : long_div(a, b);
}

// Shared items: the first key block of a range and their number, and the place
// of an item counted from the first of all.
__device__ __forceinline__ int range_begin(const PrefixSched& s, int range) { return range * s.range + min(range, s.longer); }
__device__ __forceinline__ int range_blocks(const PrefixSched& s, int range) { return s.range + (range < s.longer); }
__device__ __forceinline__ int64_t shared_place(const PrefixSched& s, int head_range, int unit) {
  return head_range * s.len_range + (int64_t)unit * s.len_two;
}

// Workspace rows: the first row of a segment; its second tile's rows follow its
// first's (tok_tile * rep of them).  Shared items come before own ones.
template <class W>
__device__ __forceinline__ int64_t shared_rows(const PrefixAttnParams& p, const PrefixSched& s, int item, int cta) {
  return ((int64_t)item + (item >= s.whole ? cta : 0)) * W::kUnitTiles * p.tok_tile * p.rep;
}
template <class W>
__device__ __forceinline__ int64_t own_rows(const PrefixAttnParams& p, const PrefixSeq& r, int unit, int head, int cta) {
  const int t0 = unit * W::kUnitTiles * p.tok_tile, tokens = min(r.rows - t0, W::kUnitTiles * p.tok_tile);
  const int64_t before = (int64_t)p.nkv * (r.first + t0) + (int64_t)head * tokens;
  const int64_t units = (int64_t)p.nkv * p.splits * p.units + p.grid + cta;
  return units * W::kUnitTiles * p.tok_tile * p.rep + before * p.rep;
}

// Four dims (chunk c) of workspace row r.  Four rows are interleaved chunk by
// chunk: a warp whose threads have a row each stores 64 contiguous bytes per four
// lanes (16 in 32 places before: the stores of a segment took 6000 cycles).
template <int HD>
__device__ __forceinline__ float4* part_chunk(float* part_o, int64_t r, int c) {
  return reinterpret_cast<float4*>(part_o) + ((r >> 2) * (HD / 4) + c) * 4 + (r & 3);
}

// The maximum of what a segment leaves (its running maximum and sum): NaN where a score was.
__device__ __forceinline__ float part_max(float2 ml) { return ml.y == ml.y ? ml.x : ml.y; }

// What a CTA works on at a time: the rows of a unit and a range of key blocks.
struct PrefixSeg {
  const int32_t* tab;   // row of the table
  int head;             // KV head
  int t0, tokens;       // rows of q
  int k0, k_end;        // keys: tokens [k0, k_end) of the sequence
  int kb0, kb1;         // blocks of them, from k0 on
  int see0;             // token i of the unit sees tokens below min(see0 + i, k_end)
  int64_t part;         // its first row of the workspace
};

__host__ __device__ constexpr uint32_t inverse_of(int x) { return (uint32_t)((((uint64_t)1 << 32) + x - 1) / x); }

// Key blocks of an item of the line (of `blocks`, each of `cost`) that belong to
// the places before `at` of it: single ones or groups, the first with the
// segment's cost, go to where they begin.
template <class W>
__device__ __forceinline__ int blocks_before(const PrefixSched& s, int64_t at, int blocks, int cost) {
  if (at <= W::kSegment) return at > 0 ? min(blocks <= kShort ? s.together : 1, blocks) : 0;
  const int together = blocks <= kShort ? s.together : 1, group = together * cost;
  const int64_t n = at - W::kSegment + group - 1;
  // n / group, by ceil(2^32 / group): exact below 2^32 / group
  constexpr int kBits = 26;
  static_assert(kTogether * (W::kFew > W::kMany ? W::kFew : W::kMany) < (1 << (32 - kBits)), "the groups' inverses");
  const uint32_t inverse = cost == W::kFew ? (together == 1 ? inverse_of(W::kFew) : inverse_of(kTogether * W::kFew))
                                           : (together == 1 ? inverse_of(W::kMany) : inverse_of(kTogether * W::kMany));
  const int64_t groups = n < (1 << kBits) ? (int64_t)__umulhi((uint32_t)n, inverse) : long_div(n, group);
  return (int)min(groups * together, (int64_t)blocks);
}

// The segments of a CTA: its whole items, and its piece [x, end) of the line.
template <class W>
struct PrefixSegs {
  const PrefixAttnParams& p;
  const PrefixSched s;
  const int64_t* line_base;
  const PrefixSeq* info;
  const int cta;
  const int32_t* shared_tab;
  int j;
  int64_t x, mid, end;                           // own segments [x, end); shared ones from mid down

  __device__ PrefixSegs(const PrefixAttnParams& p_, const PrefixSched& s_, const int64_t* base, const PrefixSeq* info_, int cta_)
      : p(p_), s(s_), line_base(base), info(info_), cta(cta_), shared_tab(nullptr), j(cta_) {
    x = piece_begin(s, cta);
    end = piece_begin(s, cta + 1);
    mid = min(end, s.shared_line);
    if (s.items > 0) {                           // base > 0: some sequence has rows
      int i = 0;
      while (i + 1 < p.n && info[i].rows == 0) ++i;
      shared_tab = p.table + (size_t)info[i].seq * p.max_pages;
    }
  }

  __device__ bool next_shared(PrefixSeg& g) {
    for (;;) {
      int gs, u, split, c0, c1;
      if (j < s.whole) {
        gs = j / p.units;
        u = j - gs * p.units;
        j += p.grid;
        split = gs % p.splits;
        c0 = 0;
        c1 = range_blocks(s, split);
      } else if (x < mid) {                      // the item of the place before mid
        const int64_t place = s.whole_line + mid - 1;
        gs = (int)div_floor(place, s.len_range);
        const int64_t rel = place - gs * s.len_range;
        u = (int)min(div_floor(rel, s.len_two), (int64_t)(p.units - 1));
        const int cost = u + 1 < p.units ? W::kMany : block_cost<W>(p, p.total - u * W::kUnitTiles * p.tok_tile);
        const int64_t to = rel - (int64_t)u * s.len_two + 1, from = max(to - (mid - x), (int64_t)0);
        mid -= to - from;
        split = gs % p.splits;
        const int blocks = range_blocks(s, split);
        c0 = blocks_before<W>(s, from, blocks, cost);
        c1 = blocks_before<W>(s, to, blocks, cost);
      } else {
        x = max(x, min(end, s.shared_line));
        return false;
      }
      if (c0 >= c1) continue;
      g.kb0 = range_begin(s, split) + c0;
      g.kb1 = range_begin(s, split) + c1;
      g.tab = shared_tab;
      g.head = gs / p.splits;
      g.t0 = u * W::kUnitTiles * p.tok_tile;
      g.tokens = min(W::kUnitTiles * p.tok_tile, p.total - g.t0);
      g.k0 = 0;
      g.k_end = g.see0 = s.base;
      g.part = shared_rows<W>(p, s, gs * p.units + u, cta);
      return true;
    }
  }

  __device__ bool next_own(PrefixSeg& g) {
    while (x < end) {
      const int64_t place = x - s.shared_line;
      int lo = 0, hi = p.n;                      // the last sequence that starts at or before it
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (line_base[mid] <= place) lo = mid; else hi = mid;
      }
      const PrefixSeq r = info[lo];
      const int units = own_units(p, r, W::kUnitTiles);
      int64_t rel = place - line_base[lo];
      int u = 0, blocks = own_blocks<W>(p, r, s.base, 0);
      int64_t len = item_length<W>(p, r, 0, blocks);
      while (rel >= len * p.nkv && u + 1 < units) {
        rel -= len * p.nkv;
        blocks = own_blocks<W>(p, r, s.base, ++u);
        len = item_length<W>(p, r, u, blocks);
      }
      if (len <= 0) break;                       // (the line is made of items that have a length)
      g.head = (int)div_floor(rel, len);
      const int64_t from = rel - g.head * len, to = min(len, from + (end - x));
      x += to - from;
      const int i0 = u * W::kUnitTiles * p.tok_tile, cost = block_cost<W>(p, r.rows - i0);
      g.kb0 = blocks_before<W>(s, from, blocks, cost);
      g.kb1 = blocks_before<W>(s, to, blocks, cost);
      if (g.kb0 >= g.kb1) continue;
      g.tab = p.table + (size_t)r.seq * p.max_pages;
      g.t0 = r.first + i0;
      g.tokens = min(W::kUnitTiles * p.tok_tile, r.rows - i0);
      g.k0 = s.base;
      g.k_end = r.len;
      g.see0 = r.len - r.rows + i0 + 1;
      g.part = own_rows<W>(p, r, u, g.head, cta);
      return true;
    }
    return false;
  }
};

}  // namespace lsp
