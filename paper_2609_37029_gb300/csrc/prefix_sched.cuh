// Work distribution of the shared-prefix attention.
//
// Query rows.  The rep = nq/nkv query heads of a KV head score the same keys,
// so a row of a tile is (token, head of the group): a tile holds tok_tile =
// tile rows / rep tokens, a unit kUnit tiles that share the keys they load.
//
// Shared part: the whole pages before every row's position that all sequences
// hold, `base` tokens.  All `total` tokens of the batch are stacked into units
// against them, without regard to whose they are (nothing is masked), and the
// keys are cut into `splits` ranges of equal size: items (head, range, unit),
// the unit fastest, dealt to the CTAs in turn, so that units of the same keys
// run at the same time and find each other's loads in L2.
//
// Own part: tokens [base, len) of each sequence, its own rows only, causal.  Its
// items, in the order (sequence, unit, head), form one line, each as long as it
// costs, that is cut into contiguous pieces so that every CTA's work, shared and
// own, adds up to about the same.  A piece may start and end inside an item.
//
// Every segment (an item, or the part of an own item that one CTA has) leaves
// unnormalised sums and the running maximum and sum of its rows in rows of the
// workspace; a second kernel joins a row's segments, which it finds by the same
// arithmetic.  Shared segments lie at
// ((head, range), unit); an own segment at (rows of the items before it) + CTA *
// (rows of a unit), which no two share: along the line the item or the CTA rises
// from segment to segment, each by at least the room of one.
#pragma once

#include <climits>

#include "common.cuh"
#include "lsp_internal.h"

namespace lsp {

struct PrefixSched {
  int base;             // tokens of the shared part
  int blocks;           // its key blocks
  int per_split;        // key blocks of a range
  int items;            // shared items
  int item_cost;        // of one, on average over the units
  int64_t own_line;     // length of the own line
};

// What work costs a CTA, for dealing it out: a key block against one and against
// two row tiles (1.1 and 1.55 us measured at 16 requests over 32K), and what a
// segment takes besides (some 2 us).
constexpr int kCostOne = 2, kCostTwo = 3, kCostSegment = 4;
template <int kUnitTiles>
__device__ __forceinline__ int block_cost(const PrefixAttnParams& p, int tokens) {
  return kUnitTiles == 1 || tokens > p.tok_tile ? kCostTwo : kCostOne;
}
struct __align__(16) PrefixSeq {
  int seq, first, rows, len;    // row of the table (-1: none), first row of q, rows, tokens
};

// Division of what outgrows 32 bits only in the longest batches, kept out of line:
// the schedule runs once, and costs what its code takes to be fetched.
static __device__ __noinline__ int64_t long_div(int64_t a, int64_t b) { return a / b; }
__device__ __forceinline__ int cdiv(int a, int b) { return (a + b - 1) / b; }

// Sequence i of the batch; rows = 0 for one the call cannot use.
__device__ __forceinline__ PrefixSeq prefix_seq(const PrefixAttnParams& p, int i, bool report) {
  PrefixSeq r;
  r.seq = p.seqs[i];
  r.first = p.start[i];
  r.rows = p.start[i + 1] - r.first;
  r.len = 0;
  const int most = p.max_pages * p.page;
  bool bad = r.first < 0 || r.rows < 0 || r.first > p.total - r.rows || r.seq < 0 || r.seq >= p.n_seqs;
  if (!bad) {
    r.len = p.len[r.seq];
    bad = r.len < 0 || r.len > most;
  }
  if (bad) {
    if (report) set_err(p.err, LSP_DEV_BAD_SEQ);
    r.seq = -1;
    r.rows = r.len = 0;
  }
  return r;
}

// Own key blocks that unit u of a sequence has to see.
template <int kUnitTiles, int kBlock>
__device__ __forceinline__ int own_blocks(const PrefixAttnParams& p, const PrefixSeq& r, int base, int u) {
  const int upto = min(r.rows, (u + 1) * kUnitTiles * p.tok_tile);
  return max(0, cdiv(r.len - r.rows + upto - base, kBlock));
}

__device__ __forceinline__ int own_units(const PrefixAttnParams& p, const PrefixSeq& r, int unit_tiles) {
  return cdiv(r.rows, unit_tiles * p.tok_tile);
}

// The own line: items of every sequence in the order (unit, head), each as long
// as it costs.  Length of an item of a unit with `blocks` key blocks:
template <int kUnitTiles>
__device__ __forceinline__ int item_length(const PrefixAttnParams& p, const PrefixSeq& r, int u, int blocks) {
  return blocks > 0 ? kCostSegment + blocks * block_cost<kUnitTiles>(p, r.rows - u * kUnitTiles * p.tok_tile) : 0;
}

// Built by one warp of every CTA; line_base [n + 1], info [n] in shared memory.
template <int kUnitTiles, int kBlock>
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
  s.blocks = cdiv(s.base, kBlock);
  s.per_split = cdiv(s.blocks, p.splits);
  s.items = s.blocks > 0 ? p.nkv * p.splits * p.units : 0;
  const int last = block_cost<kUnitTiles>(p, p.total - (p.units - 1) * kUnitTiles * p.tok_tile);
  const int64_t cost = (int64_t)s.per_split * ((p.units - 1) * kCostTwo + last);
  s.item_cost = kCostSegment + (int)(cost < INT_MAX ? (int)cost / p.units : long_div(cost, p.units));
  int64_t line = 0;
  for (int i0 = 0; i0 < p.n; i0 += 32) {
    const int i = i0 + lane;
    int64_t mine = 0;
    if (i < p.n) {
      const PrefixSeq r = info[i];               // this lane's own store
      for (int u = 0, units = own_units(p, r, kUnitTiles); u < units; ++u)
        mine += item_length<kUnitTiles>(p, r, u, own_blocks<kUnitTiles, kBlock>(p, r, s.base, u));
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
  s.own_line = line;
  return s;
}

// Where CTA c's piece of the own line begins (c == grid: the line's end).  CTAs
// below items % grid have one shared item more than the rest; the rest get as
// much of the line as a shared item costs before the others get any.  (Filling
// every CTA up by its own items' cost balances 16 requests over 32K by a few us
// more, but to find that level takes 2.4 us before anything starts.)
__device__ __forceinline__ int64_t part_of(int64_t line, int k, int n) {      // line * k / n
  return line < (1 << 21) ? (int64_t)((uint32_t)line * (uint32_t)k / (uint32_t)n) : long_div(line * k, n);   // k <= grid < 2^11
}
__device__ __forceinline__ int64_t own_begin(const PrefixSched& s, int grid, int c) {
  const int more = s.items % grid, less = grid - more;
  const int64_t fill = (int64_t)less * s.item_cost;
  if (more > 0 && s.own_line <= fill) return c <= more ? 0 : part_of(s.own_line, c - more, less);
  const int64_t even = more > 0 ? s.own_line - fill : s.own_line;
  return part_of(even, c, grid) + (more > 0 && c > more ? (int64_t)(c - more) * s.item_cost : 0);
}

// Workspace rows: the first row of a segment; its second tile's rows follow its
// first's (tok_tile * rep of them).
template <int kUnitTiles>
__device__ __forceinline__ int64_t shared_rows(const PrefixAttnParams& p, int head, int split, int unit) {
  return ((int64_t)(head * p.splits + split) * p.units + unit) * kUnitTiles * p.tok_tile * p.rep;
}
template <int kUnitTiles>
__device__ __forceinline__ int64_t own_rows(const PrefixAttnParams& p, const PrefixSeq& r, int unit, int head, int cta) {
  const int t0 = unit * kUnitTiles * p.tok_tile, tokens = min(r.rows - t0, kUnitTiles * p.tok_tile);
  const int64_t before = (int64_t)p.nkv * (r.first + t0) + (int64_t)head * tokens;
  const int64_t own0 = (int64_t)p.nkv * p.splits * p.units * kUnitTiles * p.tok_tile * p.rep;
  return own0 + before * p.rep + (int64_t)cta * kUnitTiles * p.tok_tile * p.rep;
}

// Four dims (chunk c) of workspace row r.  Four rows are interleaved chunk by
// chunk: a warp whose threads have a row each stores 64 contiguous bytes per four
// lanes (16 in 32 places before: the stores of a segment took 6000 cycles).
template <int HD>
__device__ __forceinline__ float4* part_chunk(float* part_o, int64_t r, int c) {
  return reinterpret_cast<float4*>(part_o) + ((r >> 2) * (HD / 4) + c) * 4 + (r & 3);
}

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

// Key blocks of an own item (of `blocks`, each of `cost`) that belong to the
// places before `at` of it: groups of blocks, the first with the segment's cost,
// go to where they begin.  An item cut in two is two segments, and each costs its
// CTA what a segment costs: on the tensor cores as much as two blocks, so four
// stay together; a block of the fp32 kernel takes longer than what comes with it.
template <int kUnitTiles>
__device__ __forceinline__ int blocks_before(int64_t at, int blocks, int cost) {
  constexpr int kTogether = kUnitTiles == 1 ? 1 : 4;
  if (at <= 0) return 0;
  const int group = kTogether * cost;
  const int64_t past = at - kCostSegment + group - 1;
  const int64_t groups = at <= kCostSegment ? 1 : max(past < INT_MAX ? (int64_t)((int)past / group) : long_div(past, group), (int64_t)1);
  return (int)min(groups * kTogether, (int64_t)blocks);
}

// The segments of a CTA: its shared items, and its piece [x, end) of the own line.
template <int kUnitTiles, int kBlock>
struct PrefixSegs {
  const PrefixAttnParams& p;
  const PrefixSched s;
  const int64_t* line_base;
  const PrefixSeq* info;
  const int cta;
  const int32_t* shared_tab;
  int j;
  int64_t x, end;

  __device__ PrefixSegs(const PrefixAttnParams& p_, const PrefixSched& s_, const int64_t* base, const PrefixSeq* info_, int cta_)
      : p(p_), s(s_), line_base(base), info(info_), cta(cta_), shared_tab(nullptr), j(cta_) {
    x = own_begin(s, p.grid, cta);
    end = own_begin(s, p.grid, cta + 1);
    if (s.items > 0) {                           // base > 0: some sequence has rows
      int i = 0;
      while (i + 1 < p.n && info[i].rows == 0) ++i;
      shared_tab = p.table + (size_t)info[i].seq * p.max_pages;
    }
  }

  __device__ bool next_shared(PrefixSeg& g) {
    for (; j < s.items; j += p.grid) {
      const int u = j % p.units, gs = j / p.units, split = gs % p.splits;
      g.kb0 = split * s.per_split;
      g.kb1 = min(g.kb0 + s.per_split, s.blocks);
      if (g.kb0 >= g.kb1) continue;
      g.tab = shared_tab;
      g.head = gs / p.splits;
      g.t0 = u * kUnitTiles * p.tok_tile;
      g.tokens = min(kUnitTiles * p.tok_tile, p.total - g.t0);
      g.k0 = 0;
      g.k_end = g.see0 = s.base;
      g.part = shared_rows<kUnitTiles>(p, g.head, split, u);
      j += p.grid;
      return true;
    }
    return false;
  }

  __device__ bool next_own(PrefixSeg& g) {
    while (x < end) {
      int lo = 0, hi = p.n;                      // the last sequence that starts at or before x
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (line_base[mid] <= x) lo = mid; else hi = mid;
      }
      const PrefixSeq r = info[lo];
      const int units = own_units(p, r, kUnitTiles);
      int64_t rel = x - line_base[lo];
      int u = 0, blocks = own_blocks<kUnitTiles, kBlock>(p, r, s.base, 0);
      int64_t len = item_length<kUnitTiles>(p, r, 0, blocks);
      while (rel >= len * p.nkv && u + 1 < units) {
        rel -= len * p.nkv;
        blocks = own_blocks<kUnitTiles, kBlock>(p, r, s.base, ++u);
        len = item_length<kUnitTiles>(p, r, u, blocks);
      }
      if (len <= 0) break;                       // (the line is made of items that have a length)
      g.head = rel < INT_MAX && len < INT_MAX ? (int)rel / (int)len : (int)long_div(rel, len);
      const int64_t from = rel - g.head * len, to = min(len, from + (end - x));
      x += to - from;
      const int i0 = u * kUnitTiles * p.tok_tile, cost = block_cost<kUnitTiles>(p, r.rows - i0);
      g.kb0 = blocks_before<kUnitTiles>(from, blocks, cost);
      g.kb1 = blocks_before<kUnitTiles>(to, blocks, cost);
      if (g.kb0 >= g.kb1) continue;
      g.tab = p.table + (size_t)r.seq * p.max_pages;
      g.t0 = r.first + i0;
      g.tokens = min(kUnitTiles * p.tok_tile, r.rows - i0);
      g.k0 = s.base;
      g.k_end = r.len;
      g.see0 = r.len - r.rows + i0 + 1;
      g.part = own_rows<kUnitTiles>(p, r, u, g.head, cta);
      return true;
    }
    return false;
  }
};

}  // namespace lsp
