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
// Own part: tokens [base, len) of each sequence, its own rows only, causal.
// Its key blocks, in the order (sequence, unit, head, block), form one line of
// `own_steps` steps that is cut into contiguous pieces so that every CTA's
// blocks, shared and own, add up to about the same number.  A piece may start
// and end inside an item.
//
// Every segment (an item, or the part of an own item that one CTA has) leaves
// unnormalised sums and the running maximum and sum of its rows in rows of the
// workspace; a second kernel joins a row's segments.  Shared segments lie at
// ((head, range), unit); an own segment at kUnit * (rows of the items before
// it) + CTA * (rows of a unit), which no two share: along the line the item or
// the CTA rises from segment to segment, each by at least the room of one.
#pragma once

#include "common.cuh"
#include "lsp_internal.h"

namespace lsp {

struct PrefixSched {
  int base;             // tokens of the shared part
  int blocks;           // its key blocks
  int per_split;        // key blocks of a range
  int items;            // shared items
  int64_t own_steps;    // key blocks of the own part
};
// The schedule in the workspace: PrefixSched, then the first own step of each sequence.
constexpr size_t kSchedHdrBytes = 32;

struct PrefixSeq {
  int seq, first, rows, len;    // row of the table (-1: none), first row of q, rows, tokens
};

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

// Built by one warp of every CTA; step_base: [n + 1] in shared memory.
template <int kUnitTiles, int kBlock>
__device__ __forceinline__ PrefixSched build_sched(const PrefixAttnParams& p, int64_t* step_base, bool report) {
  const int lane = threadIdx.x & 31;
  PrefixSched s;
  int base = p.shared_len;
  for (int i = lane; i < p.n; i += 32) {
    const PrefixSeq r = prefix_seq(p, i, report);
    if (r.rows > 0) base = min(base, r.len - r.rows);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) base = min(base, __shfl_xor_sync(0xffffffffu, base, o));
  s.base = max(base, 0) / p.page * p.page;
  s.blocks = cdiv(s.base, kBlock);
  s.per_split = cdiv(s.blocks, p.splits);
  s.items = s.blocks > 0 ? p.nkv * p.splits * p.units : 0;
  int64_t steps = 0;
  for (int i0 = 0; i0 < p.n; i0 += 32) {
    const int i = i0 + lane;
    int64_t mine = 0;
    if (i < p.n) {
      const PrefixSeq r = prefix_seq(p, i, false);
      for (int u = 0, units = own_units(p, r, kUnitTiles); u < units; ++u)
        mine += own_blocks<kUnitTiles, kBlock>(p, r, s.base, u);
      mine *= p.nkv;
    }
    int64_t x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t a = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += a;
    }
    if (i < p.n) step_base[i] = steps + x - mine;
    steps += __shfl_sync(0xffffffffu, x, 31);
  }
  if (lane == 0) step_base[p.n] = steps;
  s.own_steps = steps;
  return s;
}

// First own step of CTA c (c == grid: the end).  CTAs below items % grid have
// one shared item more than the rest; the rest get per_split own steps before
// the others get any.
__device__ __forceinline__ int64_t own_begin(const PrefixSched& s, int grid, int c) {
  const int more = s.items % grid, less = grid - more;
  const int64_t fill = (int64_t)less * s.per_split;
  if (more > 0 && s.own_steps <= fill) return c <= more ? 0 : s.own_steps * (c - more) / less;
  const int64_t even = more > 0 ? s.own_steps - fill : s.own_steps;
  return even * c / grid + (more > 0 && c > more ? (int64_t)(c - more) * s.per_split : 0);
}

// Where a step of the own line lies.
struct OwnSpot {
  int i, unit, head, blocks, block;
};
template <int kUnitTiles, int kBlock>
__device__ __forceinline__ OwnSpot own_spot(const PrefixAttnParams& p, const PrefixSched& s, const int64_t* step_base,
                                            int64_t step) {
  int lo = 0, hi = p.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (step_base[mid] <= step) lo = mid; else hi = mid;
  }
  const PrefixSeq r = prefix_seq(p, lo, false);
  const int units = own_units(p, r, kUnitTiles);
  int64_t rel = step - step_base[lo];
  OwnSpot o;
  o.i = lo;
  o.unit = 0;
  o.blocks = own_blocks<kUnitTiles, kBlock>(p, r, s.base, 0);
  while (rel >= (int64_t)o.blocks * p.nkv && o.unit + 1 < units) {
    rel -= (int64_t)o.blocks * p.nkv;
    o.blocks = own_blocks<kUnitTiles, kBlock>(p, r, s.base, ++o.unit);
  }
  o.head = (int)(rel / max(o.blocks, 1));
  o.block = (int)(rel - (int64_t)o.head * o.blocks);
  return o;
}

// Workspace rows: the first row of a segment, and where its second tile (or the
// second stream of a unit with one tile) starts.
struct PartRows {
  int64_t row;
  int second;
};
template <int kUnitTiles>
__device__ __forceinline__ PartRows shared_rows(const PrefixAttnParams& p, int head, int split, int unit) {
  const int tile = p.tok_tile * p.rep;
  return {((int64_t)(head * p.splits + split) * p.units + unit) * kUnitTiles * tile, tile};
}
template <int kUnitTiles>
__device__ __forceinline__ PartRows own_rows(const PrefixAttnParams& p, const PrefixSeq& r, int unit, int head, int cta) {
  const int t0 = unit * kUnitTiles * p.tok_tile, tokens = min(r.rows - t0, kUnitTiles * p.tok_tile);
  const int64_t before = (int64_t)p.nkv * (r.first + t0) + (int64_t)head * tokens;
  const int64_t own0 = (int64_t)p.nkv * p.splits * p.units * kUnitTiles * p.tok_tile * p.rep;
  return {own0 + kUnitTiles * (before * p.rep + (int64_t)cta * p.tok_tile * p.rep), min(tokens, p.tok_tile) * p.rep};
}

}  // namespace lsp
